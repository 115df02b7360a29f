// Norms of queries and keys for each head and the rotation by position, in one pass over both tensors.
//   y = x w / sqrt(mean(x^2) + eps);   (a, b) -> (a cos - b sin, b cos + a sin), angle = position * freq
// It lives on memory bandwidth: every row is read once and written once, 16 lanes a row, eight columns a lane.
// All heads of a token turn by the same angles; a workgroup takes 16 heads of four tokens, makes the four
// tables meanwhile its 64 rows are on their way (a wave a token, a lane a frequency), and each lane turns four
// rows of one token.  8 x 4096 tokens x 32 + 32 heads, bf16, 1.07 GB: 190 us, 5.6 TB/s (a copy: 4.8); with all
// heads of a token in one workgroup, row after row, 268.  One token x 32 + 8 heads: 2.8 us against 11.
#include "decode_device.h"
#include "tf_kernels.h"

namespace tf {

namespace {

// STREAM: past the caches
template <bool STREAM>
__device__ __forceinline__ void put16(void* p, u32x4 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
    else *static_cast<u32x4*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ void store_row(uint16_t* p, const float* x)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        r[i] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});   // to nearest even
    }
    put16<STREAM>(p, r);
}
template <bool STREAM>
__device__ __forceinline__ void store_row(float* p, const float* x)
{
    put16<STREAM>(p, __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}));
    put16<STREAM>(p + 4, __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}));
}

// A workgroup takes TOKENS tokens and 16 heads of one of the tensors.
template <typename T, int TOKENS, bool STREAM>
__global__ __launch_bounds__(256) void norm_rotate_kernel(const NormRotateArgs a)
{
    constexpr int kRows = TOKENS;   // of a lane
    __shared__ float2 turn[TOKENS][64];   // cos, sin
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int groups = (a.n + TOKENS - 1) / TOKENS;
    const int part = blockIdx.x % a.parts, at = blockIdx.x / a.parts;
    const int b = at / groups, t0 = at % groups * TOKENS, half = a.rot_dim / 2;
    const bool is_k = part >= a.parts_q;
    const int h0 = 16 * (is_k ? part - a.parts_q : part), heads = is_k ? a.Hkv : a.Hq;
    const long long s_b = is_k ? a.kvs[0] : a.qs[0], s_h = is_k ? a.kvs[1] : a.qs[1], s_t = is_k ? a.kvs[2] : a.qs[2];
    const long long o_b = is_k ? a.kvs[0] : a.os[0], o_h = is_k ? a.kvs[1] : a.os[1], o_t = is_k ? a.kvs[2] : a.os[2];
    const T* const src = static_cast<const T*>(is_k ? a.K : a.Q) + b * s_b + 8 * l16;
    T* const dst = static_cast<T*>(is_k ? a.K_out : a.Q_out) + b * o_b + 8 * l16;
    const float* const w = is_k ? a.k_weight : a.q_weight;
    // a lane's rows are one token's; the four rows of a wave lie side by side in memory
    const bool by_head = s_h < s_t;
    const int tok = TOKENS == 1 ? 0 : by_head ? grp / 4 : grp % 4;
    const int h_first = h0 + (TOKENS == 1 ? grp : by_head ? grp % 4 : grp / 4);
    const int t = min(t0 + tok, a.n - 1);
    float x[kRows][8];
#pragma unroll
    for (int u = 0; u < kRows; ++u) load8(src + min(h_first + 4 * u, heads - 1) * s_h + t * s_t, x[u]);
    float wt[8];
    if (w) load8(w + 8 * l16, wt);

    if (wave < TOKENS && lane < half) {
        const int tw = min(t0 + wave, a.n - 1);
        const long long pos = (long long)(a.positions ? a.positions[(long long)b * a.n + tw] : tw) + (a.start ? a.start[b] : 0);
        // whole turns are taken off in 64 bits: what is left of a far position's angle has no error to speak of
        double turns = (double)pos * a.freq[lane] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        turn[wave][lane] = make_float2(c, s);
    }
    __syncthreads();
    // (a, b) of a pair lie in one lane, or `half` columns apart
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int col = 8 * l16 + i;
        const float2 r = turn[tok][col >= a.rot_dim ? 0 : a.interleaved ? col / 2 : col < half ? col : col - half];
        const bool second = a.interleaved ? col & 1 : col >= half;
        cs[i] = r.x;
        sn[i] = second ? r.y : -r.y;
    }
    const bool turned = 8 * l16 < a.rot_dim;   // (rot_dim is a multiple of 16: all of a lane's columns or none)
    const int hop = half / 8, mate = !turned ? l16 : l16 < hop ? l16 + hop : l16 - hop;
    const int from = (lane & 48) + mate;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int h = h_first + 4 * u;
        if (w) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[u][i], x[u][i], ss);
            const float r = 1.0f / sqrtf(row16_sum(ss) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = x[u][i] * r * wt[i];
        }
        float y[8];
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(x[u][i], cs[i], x[u][i ^ 1] * sn[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(x[u][i], cs[i], __shfl(x[u][i], from) * sn[i]);
        }
        // (no arithmetic for what is passed on: by cos 1 and sin 0 an infinity would become a NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = turned ? y[i] : x[u][i];
        if (h < heads && t0 + tok < a.n) store_row<STREAM>(dst + h * o_h + t * o_t, y);
    }
}

}  // namespace

// Where four tokens a workgroup leave no more than two on a compute unit, one each: latency counts there
// (32 + 8 heads, 16 / 200 / 1000 / 2048 tokens: 4.7, 4.9, 8.5, 12.5 us by fours, 3.4, 4.2, 9.0, 13.8 one by one).
static bool one_by_one(const NormRotateArgs& a) { return a.n < 4 || (long long)a.B * a.n * a.parts <= 4 * 512; }

long long norm_rotate_workgroups(NormRotateArgs& a)
{
    a.parts_q = a.Q ? (a.Hq + 15) / 16 : 0;
    a.parts = a.parts_q + (a.K ? (a.Hkv + 15) / 16 : 0);
    return (long long)a.parts * a.B * (one_by_one(a) ? a.n : (a.n + 3) / 4);
}

hipError_t launch_norm_rotate(const NormRotateArgs& in, int dtype, hipStream_t s)
{
    NormRotateArgs a = in;
    const unsigned grid = (unsigned)norm_rotate_workgroups(a);
    const bool few = one_by_one(a);
    const long long rows = (long long)a.B * a.n;
    // Results that would push everything out of the 256 MB cache behind the L2s go past it (the case above
    // 206 us without); smaller ones are what the next call reads.
    const bool stream = (dtype == 0 ? 8 : 4) * rows * kHeadDim * ((a.Q ? a.Hq : 0) + (a.K ? a.Hkv : 0)) > (256ll << 20);
#define TF_NORM_ROTATE(T)                                                                          \
    do {                                                                                          \
        if (few) norm_rotate_kernel<T, 1, false><<<dim3(grid), dim3(256), 0, s>>>(a);             \
        else if (stream) norm_rotate_kernel<T, 4, true><<<dim3(grid), dim3(256), 0, s>>>(a);      \
        else norm_rotate_kernel<T, 4, false><<<dim3(grid), dim3(256), 0, s>>>(a);                 \
    } while (0)
    if (dtype == 0) TF_NORM_ROTATE(float);
    else TF_NORM_ROTATE(uint16_t);
#undef TF_NORM_ROTATE
    return hipGetLastError();
}

}  // namespace tf
