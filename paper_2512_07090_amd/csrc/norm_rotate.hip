// Norms of queries and keys for each head and the rotation by position, in one pass over both tensors.
//   y = x w / sqrt(mean(x^2) + eps);   (a, b) -> (a cos - b sin, b cos + a sin), angle = position * freq
// It lives on memory bandwidth: every row is read once and written once, 16 lanes a row, eight columns a lane.
// All heads of a token turn by the same angles, so a workgroup takes four tokens with all their heads and makes
// each token's table once, a wave a token, a lane a frequency.
#include "decode_device.h"
#include "tf_kernels.h"

namespace tf {

namespace {

constexpr int kTokens = 4;   // of a workgroup: one table a wave

__device__ __forceinline__ void store_row(uint16_t* p, const float* x)
{
    uint4 r;
    unsigned* w = reinterpret_cast<unsigned*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const bf16x2 v = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};   // to nearest even
        w[i] = __builtin_bit_cast(unsigned, v);
    }
    *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store_row(float* p, const float* x)
{
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

template <typename T>
__global__ __launch_bounds__(256) void norm_rotate_kernel(const NormRotateArgs a)
{
    __shared__ float2 turn[kTokens][64];   // cos, sin
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int groups = (a.n + kTokens - 1) / kTokens;
    const int b = blockIdx.x / groups, t0 = blockIdx.x % groups * kTokens, half = a.rot_dim / 2;
    if (lane < half && t0 + wave < a.n) {
        const int t = t0 + wave;
        const long long pos = (long long)(a.positions ? a.positions[(long long)b * a.n + t] : t) + (a.start ? a.start[b] : 0);
        // whole turns are taken off in 64 bits: what is left of a far position's angle has no error to speak of
        double turns = (double)pos * a.freq[lane] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        turn[wave][lane] = make_float2(c, s);
    }
    __syncthreads();
    const int grp = threadIdx.x >> 4, l16 = threadIdx.x & 15;
    const int t = t0 + (grp & (kTokens - 1));
    if (t >= a.n) return;
    const int heads_q = a.Q ? a.Hq : 0, heads = heads_q + (a.K ? a.Hkv : 0);
    // (a, b) of a pair lie in one lane, or `half` columns apart
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int col = 8 * l16 + i;
        const float2 r = col >= a.rot_dim ? make_float2(1.f, 0.f)
                       : turn[grp & (kTokens - 1)][a.interleaved ? col / 2 : col < half ? col : col - half];
        const bool second = a.interleaved ? col & 1 : col >= half;
        cs[i] = r.x;
        sn[i] = second ? r.y : -r.y;
    }
    const int hop = half / 8, mate = 8 * l16 >= a.rot_dim ? l16 : l16 < hop ? l16 + hop : l16 - hop;
    const int from = (lane & 48) + mate;
    for (int h = grp / kTokens; h < heads; h += 16 / kTokens) {
        const bool is_k = h >= heads_q;
        const int hh = is_k ? h - heads_q : h;
        const long long* const st = is_k ? a.kvs : a.qs;
        const long long* const so = is_k ? a.kvs : a.os;
        const T* const src = static_cast<const T*>(is_k ? a.K : a.Q) + b * st[0] + hh * st[1] + t * st[2] + 8 * l16;
        T* const dst = static_cast<T*>(is_k ? a.K_out : a.Q_out) + b * so[0] + hh * so[1] + t * so[2] + 8 * l16;
        const float* const w = is_k ? a.k_weight : a.q_weight;
        float x[8];
        load8(src, x);
        if (w) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
            const float r = 1.0f / sqrtf(row16_sum(ss) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[8 * l16 + i];
        }
        float y[8];
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(x[i], cs[i], x[i ^ 1] * sn[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(x[i], cs[i], __shfl(x[i], from) * sn[i]);
        }
        store_row(dst, y);
    }
}

}  // namespace

hipError_t launch_norm_rotate(const NormRotateArgs& a, int dtype, hipStream_t s)
{
    const unsigned grid = (unsigned)a.B * (unsigned)((a.n + kTokens - 1) / kTokens);
    if (dtype == 0) norm_rotate_kernel<float><<<dim3(grid), dim3(256), 0, s>>>(a);
    else norm_rotate_kernel<uint16_t><<<dim3(grid), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace tf
