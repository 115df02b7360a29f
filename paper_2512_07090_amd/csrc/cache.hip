// A cache in 4 or 8 bits (the format: cache_format.h): rows quantised as they are written, read back, and
// attended to by the new tokens of a sequence.
#include <algorithm>
#include <type_traits>

#include "cache_format.h"
#include "decode_device.h"
#include "tf_kernels.h"

namespace tf {

namespace {

constexpr int kPartStride = kDecodePartFloats;
constexpr float kNoKey = -3.0e38f;   // the maximum of no scores: below all of them, and finite, so differences of two are 0

// STREAM: past the caches
template <bool STREAM>
__device__ __forceinline__ void put16(void* p, u32x4 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
    else *static_cast<u32x4*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ void store8(uint16_t* p, const float* x)
{
    u32x4 r;   // (what a code stands for is exact in bf16 down to 2^-133)
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
    put16<STREAM>(p, r);
}
template <bool STREAM>
__device__ __forceinline__ void store8(float* p, const float* x)
{
    put16<STREAM>(p, __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}));
    put16<STREAM>(p + 4, __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}));
}

// eight elements of a row that is not needed again, past the caches
__device__ __forceinline__ void stream8(const uint16_t* p, float* x)
{
    const u32x4 r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void stream8(const float* p, float* x)
{
    const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}

// position of the j-th row that is written (one outside of the sequence is the caller's mistake; it is not read from there)
__device__ __forceinline__ int position(const CacheWriteArgs& a, int b, int j)
{
    return a.kept_idx ? min(max(a.kept_idx[(long long)b * a.m + j], 0), a.n - 1) : j;
}

// A workgroup takes one page of one (tensor, batch row, KV head): 16 lanes a row, four rows a lane, all of which
// are requested before the first is used.  It lives on memory bandwidth: 8 x 32 heads x 2048 of 4096 rows, bf16
// to 4 bits, 340 MB: 66 us, 5.1 TB/s; with loads that stay in the caches 89, with keys and values of a page in
// one workgroup 68.
template <typename T, int BITS>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheWriteArgs a)
{
    const int w = blockIdx.x & 1, rest = blockIdx.x >> 1;
    const int page_i = rest % a.pages, bh = rest / a.pages, b = bh / a.Hkv, h = bh % a.Hkv;
    const int held = min(max(a.len[b], 0), a.capacity);
    const int rows = min(a.count ? min(max(a.count[b], 0), a.m) : a.m, a.capacity - held);
    const int page = held / kPageRows + page_i;
    if (rows < 1 || page * kPageRows >= held + rows) return;
    const int c = threadIdx.x & 15, grp = threadIdx.x >> 4;
    float x[4][8];
    bool there[4];
    int t[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = page * kPageRows + 16 * u + grp - held;   // the i-th row that is written
        there[u] = i >= 0 && i < rows;
        t[u] = position(a, b, min(max(i, 0), rows - 1));
    }
    const T* const src = static_cast<const T*>(w ? a.V : a.K) + b * a.kvs[0] + h * a.kvs[1] + 8 * c;
#pragma unroll
    for (int u = 0; u < 4; ++u) stream8(src + t[u] * a.kvs[2], x[u]);
    uint8_t* const dst = static_cast<uint8_t*>(w ? a.v : a.k) + ((long long)bh * a.cache_pages + page) * page_bytes<BITS>();
#pragma unroll
    for (int u = 0; u < 4; ++u) store_row8<BITS>(dst, 16 * u + grp, c, x[u], w, there[u]);
}

// len and overflow once the rows are written; a row's old length is read by all of its workgroups, so this is a
// launch of its own
__device__ __forceinline__ void advance(const CacheWriteArgs& a, int b, int held)
{
    const int rows = a.count ? min(max(a.count[b], 0), a.m) : a.m;
    a.len[b] = held + min(rows, a.capacity - held);
    if (a.overflow && rows > a.capacity - held) a.overflow[b] = 1;
}
__global__ void cache_advance_kernel(const CacheWriteArgs a)
{
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < a.B) advance(a, b, min(max(a.len[b], 0), a.capacity));
}

// A few new rows (a decoded token's): one workgroup writes all of a batch row's and moves its length on, in one
// launch (8 x 8 KV heads x 1 row: 3 us against 3 + 2 and the launch).
constexpr int kAppendRows = 256;   // rows of keys and values of all heads: four a lane
template <typename T, int BITS>
__global__ __launch_bounds__(1024) void cache_append_kernel(const CacheWriteArgs a)
{
    const int b = blockIdx.x, c = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int held = min(max(a.len[b], 0), a.capacity);
    const int rows = min(a.count ? min(max(a.count[b], 0), a.m) : a.m, a.capacity - held);
    const int jobs = 2 * a.Hkv * rows;   // row i of head h, keys first
    float x[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int job = grp + 64 * u;
        if (job >= jobs) break;
        const int i = job % rows, wh = job / rows, w = wh >= a.Hkv, h = wh - w * a.Hkv;
        stream8(static_cast<const T*>(w ? a.V : a.K) + b * a.kvs[0] + h * a.kvs[1] + position(a, b, i) * a.kvs[2] + 8 * c, x[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int job = grp + 64 * u;
        if (job >= jobs) break;
        const int i = job % rows, wh = job / rows, w = wh >= a.Hkv, h = wh - w * a.Hkv, slot = held + i;
        uint8_t* const page = static_cast<uint8_t*>(w ? a.v : a.k) + (((long long)b * a.Hkv + h) * a.cache_pages + slot / kPageRows) * page_bytes<BITS>();
        store_row8<BITS>(page, slot % kPageRows, c, x[u], w, true);
    }
    __syncthreads();   // every thread has read the old length
    if (threadIdx.x == 0) advance(a, b, held);
}

// The reverse, rows start[b] .. start[b] + n - 1 of the cache; the same 2048 rows of 8 x 32 heads: 59 us, 50 (6.8 TB/s)
// with stores past the caches.
template <typename T, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheReadArgs a)
{
    const int w = blockIdx.x & 1, rest = blockIdx.x >> 1;
    const int page_i = rest % a.pages, bh = rest / a.pages, b = bh / a.Hkv, h = bh % a.Hkv;
    const int held = min(max(a.len[b], 0), a.capacity), from = a.start ? max(a.start[b], 0) : 0;
    if (from >= held) return;
    const int to = min(held, from + min(a.n, held - from)), page = from / kPageRows + page_i;
    if (page * kPageRows >= to) return;
    T* const dst = static_cast<T*>(w ? a.V : a.K) + b * a.kvs[0] + h * a.kvs[1];
    const uint8_t* const src = static_cast<const uint8_t*>(w ? a.v : a.k) + ((long long)bh * a.cache_pages + page) * page_bytes<BITS>();
    const int c = threadIdx.x & 15, grp = threadIdx.x >> 4;
    unsigned code[4][BITS / 4];
    int e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {   // (a page is there as a whole)
        const int row = 16 * u + grp;
        const unsigned* at = reinterpret_cast<const unsigned*>(src + (w ? value_code_at<BITS>(row, c) : key_code_at<BITS>(row, c)));
#pragma unroll
        for (int i = 0; i < BITS / 4; ++i) code[u][i] = at[i];
        e[u] = src[w ? value_scale_at<BITS>(row, c >> 2) : key_scale_at<BITS>(row, c >> 2)];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int slot = page * kPageRows + 16 * u + grp;
        if (slot < from || slot >= to) continue;
        float x[8];
        values_of8<BITS>(code[u], exponent_scale(e[u]), x);
        store8<STREAM>(dst + (slot - from) * a.kvs[2] + 8 * c, x);
    }
}

__device__ __forceinline__ void store_pair(uint16_t* p, float x, float y)
{
    *reinterpret_cast<unsigned*>(p) = __builtin_bit_cast(unsigned, bf16x2{(__bf16)x, (__bf16)y});
}
__device__ __forceinline__ void store_pair(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }

// ---- attention -----------------------------------------------------------------------------
// A column is one query of one head: token t, head g of the `ratio` that share a KV head, column t * ratio + g.
// A workgroup takes CT tiles of 16 columns and one slice of the row's keys, a wave a page of 64 keys at a time.
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, A: 16 keys, B: the columns.  A lane holds a block of 32 columns of a
//                 key (the contraction order is dealt out so that these are contiguous), with one scale.
//   O^T += V^T P^T  A: eight columns of the eight keys whose weights the lane holds, transposed within the lane.
// Codes become bf16 exactly, two an instruction.  fp32 queries and their weights are sums of three bf16 parts, which
// is exact.  Behind bf16 queries weights are two parts (2^-16), or, where a call has many columns (CT = 2), rounded
// to bf16 once as the batched attention does, numerator and denominator alike: with two parts 2 x 256 queries of 32
// / 8 heads x 6000 keys took 85 us, 68 so.  Up to eight columns leave room for the second parts as columns of their
// own (PAIRED: column c16 % 8, part c16 / 8), which halves the second product: 64 / 8 heads x 4000 14.2 -> 13.6 us,
// 32 / 8 x 500 6.6 -> 6.4, 16 x 32 / 8 x up to 16384 50.4 -> 49.6.
// (The scaled 4-bit product, which would take codes as they are, adds up with less than fp32: 1.5e-4 of the sum of
// magnitudes was measured, and queries would have to be rounded to 8 bits.)
// What bounds it: long caches the way of their bytes (8 x 32 heads x 8192 keys in 4 bits, 285 MB: 51 us, 5.6 TB/s),
// many queries the vector unit and the matrix pipe, mostly in turn: 2 x 256 queries x 6000 keys, 40.7 GFLOP, 59 us, 9.2
// to 10 us for each 1024 keys more, which is 0.86 to 0.93 PFLOP/s where a large library product reaches 1.25; vector
// instructions are under way 56 % of the time, matrix ones 30 %, 65 and 35 % in 4 x 512 x 8000 (of 57 us once, without
// exponentials 54.5, without converting codes 53).  Between them every tile of 16 columns converts a cache's pages again:
// 64 queries x 8000 keys 24.5 us, 51 and 20 %.  Short caches are a chain of latencies (32 / 8 heads x 500 keys: 5.9 us, of
// which a launch with one load takes 2.5).

// Parts of two values: three of them cut off, which is exact, or two rounded.
template <int PARTS>
__device__ __forceinline__ void split_pair(float a, float b, unsigned* w)
{
    if constexpr (PARTS == 1) {
        w[0] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
    } else if constexpr (PARTS == 3) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            w[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
            a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
    } else {
        w[0] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
        w[1] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)(a - __uint_as_float(w[0] << 16)), (__bf16)(b - __uint_as_float(w[0] & 0xffff0000u))});
    }
}
template <int PARTS>
__device__ __forceinline__ void load_query(const uint16_t* p, bf16x8* f)
{
    static_assert(PARTS == 1, "bf16 queries are whole");
    f[0] = *reinterpret_cast<const bf16x8*>(p);
}
template <int PARTS>
__device__ __forceinline__ void load_query(const float* p, bf16x8* f)
{
    float x[8];
    load8(p, x);
    u32x4 r[PARTS];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned w[PARTS];
        split_pair<PARTS>(x[2 * i], x[2 * i + 1], w);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) r[k][i] = w[k];
    }
#pragma unroll
    for (int k = 0; k < PARTS; ++k) f[k] = __builtin_bit_cast(bf16x8, r[k]);
}

template <typename T, int BITS, int CT, int WAVES, bool PAIRED>
__global__ __launch_bounds__(64 * WAVES, 2) void cache_attend_kernel(const CacheAttendArgs a)
{
    static_assert(!PAIRED || (sizeof(T) == 2 && CT == 1), "");
    constexpr int kQ = sizeof(T) == 2 ? 1 : 3, kP = PAIRED ? 1 : sizeof(T) != 2 ? 3 : CT == 1 ? 2 : 1;   // bf16 parts of a query, of a weight
    constexpr bool kWholeSum = PAIRED || kP > 1;   // denominators from the weights before they are rounded
    constexpr int kRaw = BITS / 4;                                            // 16-byte loads of a lane and tile
    constexpr int kCols = 16 * CT, kThreads = 64 * WAVES, kRow = kHeadDim + 4;
    __shared__ __attribute__((aligned(16))) float o_part[WAVES][kCols][kRow];
    __shared__ float stat[WAVES][kCols][2];
    __shared__ int drawn;
    const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // The tiles of a cache go to one die, whose L2 they then share: workgroups are dealt out to the dies in turn, so
    // eight caches a time, one for each; what is left over of them is spread.
    int at = blockIdx.x;
    int bh = quotient(quotient(at, a.by_split), a.by_tiles);
    if (a.tiles > 1) {
        const int group = a.n_split * a.tiles, eight = bh >> 3;
        if (8 * eight + 8 <= a.B * a.Hkv) {
            const int in = at - 8 * eight * group;
            bh = 8 * eight + (in & 7);
            at = in >> 3;
        }
    }
    const int slice_of = quotient(at, a.by_split), sp = at - slice_of * a.n_split;
    const int tile = slice_of - quotient(slice_of, a.by_tiles) * a.tiles;
    const int b = quotient(bh, a.by_hkv), hk = bh - b * a.Hkv;
    const int ratio = a.by_ratio.by;
    const int held = min(max(a.len[b], 0), a.capacity);
    const int there = a.skip && a.skip[b] ? 0 : a.count ? min(max(a.count[b], 0), a.n) : a.n;   // queries of this row
    // keys that query t sees (none: a zero row)
    auto sees = [&](int t) { return t < there ? max(held - there + t + 1, 0) : 0; };
    const int cols = min(kCols, a.n * ratio - tile * kCols);
    auto token = [&](int col) { return quotient(tile * kCols + col, a.by_ratio); };
    const int first_t = token(0), last_t = min(token(cols - 1), there - 1);
    const int keys = last_t < first_t ? 0 : sees(last_t);        // of any of the columns
    T* const out = static_cast<T*>(a.o) + b * a.os[0];
    auto out_row = [&](int col) {
        const int q = tile * kCols + col, t = quotient(q, a.by_ratio);
        return out + (hk * ratio + q - t * ratio) * a.os[1] + t * a.os[2];
    };
    // The slices of a row follow from its own length.  Up to 512 keys are one (500 keys: 8.1 us in two, 6.7 in one then),
    // rows of up to 16384 at most 16, whose merge costs less than 32 compute units bring, and longer ones up to n_split
    // (kDecodeMaxSplit at most) of 1024 keys or more: of 256, 512, 1024 keys 1 x 32 / 8 heads x 4000 keys 8.1, 8.1, 9.1 us;
    // 8000 10.7, 9.2, 9.3; 16000 12.4, 12.4, 11.1; 8 / 1 heads x 4000 7.7, 8.4, 9.4.
    const int least = held <= 512 ? 512 : held <= 4096 ? 256 : held <= 8192 ? 512 : 1024;
    const int chunk = max(least, (quotient(held + a.n_split - 1, a.by_split) + kPageRows - 1) / kPageRows * kPageRows);
    const int used = (keys + chunk - 1) / chunk;
    if (sp >= used) {
        if (used == 0 && sp == 0)
            for (int i = threadIdx.x; i < cols * kHeadDim; i += kThreads) store_out(out_row(i / kHeadDim) + i % kHeadDim, 0.f);
        return;
    }
    const int lo = sp * chunk, hi = min(keys, lo + chunk);
    const int all_see = sees(first_t);   // keys that every column sees

    // The ticket of these columns counts the slices that are done, of this call: its upper bits are the call's own
    // number, set by whoever finds another there (whatever it is: the workspace comes as it is).
    unsigned long long* const ticket = a.tickets + bh * a.tiles + tile;
    if (used > 1 && threadIdx.x == 0) {
        unsigned long long old = __hip_atomic_load(ticket, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (old >> 16 != a.call)
            __hip_atomic_compare_exchange_strong(ticket, &old, a.call << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }

    bf16x8 qf[kQ][CT][4];
    int my_keys[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int col = min(16 * ct + (PAIRED ? c16 % 8 : c16), cols - 1), q = tile * kCols + col, t = quotient(q, a.by_ratio);
        my_keys[ct] = sees(t);
        const T* const row = static_cast<const T*>(a.q) + b * a.qs[0] + (hk * ratio + q - t * ratio) * a.qs[1] + t * a.qs[2] + 32 * g4;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf16x8 f[kQ];
            load_query<kQ>(row + 8 * s, f);
#pragma unroll
            for (int i = 0; i < kQ; ++i)
                qf[i][ct][s] = f[i];
        }
    }
    const long long row_at = (long long)bh * a.cache_pages * page_bytes<BITS>();
    const uint8_t* const kb = static_cast<const uint8_t*>(a.k) + row_at;
    const uint8_t* const vb = static_cast<const uint8_t*>(a.v) + row_at;

    const float second = PAIRED && c16 >= 8 ? -1.f : 0.f;
    f32x4 acc[CT][8];
    float mx[CT], sum[CT];
    f32x4 total[CT];   // (with whole weights: their sums on the matrix pipe, as rounded, in every register)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        mx[ct] = kNoKey; sum[ct] = 0.f;
        total[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    u32x4 k_raw[4][kRaw], v_raw[4][kRaw], v_scale;
    unsigned k_scale;
    auto request_k = [&](int j) {
        const uint8_t* p = kb + (long long)(j / kPageRows) * page_bytes<BITS>();
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < kRaw; ++i) k_raw[t][i] = *reinterpret_cast<const u32x4*>(p + key_code_at<BITS>(16 * t + c16, 4 * g4) + 16 * i);
        k_scale = *reinterpret_cast<const unsigned*>(p + page_codes<BITS>() + 4 * lane);
        asm volatile("" ::: "memory");   // (the compiler moves these loads to where they are used)
    };
    auto request_v = [&](int j) {
        const uint8_t* p = vb + (long long)(j / kPageRows) * page_bytes<BITS>();
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < kRaw; ++i) v_raw[t][i] = *reinterpret_cast<const u32x4*>(p + value_code_at<BITS>(16 * t + 4 * g4, c16) + 16 * i);
        v_scale = *reinterpret_cast<const u32x4*>(p + page_codes<BITS>() + (4 * g4 + (c16 >> 2)) * 16);
        asm volatile("" ::: "memory");
    };
    // A wave's page; `more`: another one follows, whose codes are requested as soon as this one's are used up.  (As a
    // condition in the loop the requests made every wait one for all of them: 16 x 32 / 8 x up to 16384 48.4 us, 46.2 so.)
    auto weigh_page = [&](int j, auto more) {
        // scores of the page, a tile of 16 keys after the other
        float s[CT][16], factor[CT];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float scale = exponent_scale((k_scale >> (8 * t)) & 0xff);
            f32x4 d[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) d[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                unsigned code[BITS / 4];
#pragma unroll
                for (int i = 0; i < BITS / 4; ++i) code[i] = k_raw[t][(BITS / 4 * st + i) / 4][(BITS / 4 * st + i) % 4];
                u32x4 f;
                unsigned pair[4];
                bf16_of8<BITS>(code, scale, pair);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = pair[i];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < kQ; ++i) d[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), qf[i][ct][st], d[ct], 0, 0, 0);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int v = 0; v < 4; ++v) s[ct][4 * t + v] = d[ct][v];
        }
        if constexpr (more) request_k(j + WAVES * kPageRows);
        if (j + kPageRows > all_see) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (j + 16 * t + 4 * g4 + v >= my_keys[ct]) s[ct][4 * t + v] = -INFINITY;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float top = s[ct][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[ct][i]);
            top = wave_group_max(top) * a.scale_log2e;
            // (a reference that lags behind by up to 8 leaves weights of up to 256, and the sums are left alone: moved with
            // every new maximum, one of a wave's columns has one in most pages: 2 x 256 queries 67.5 us, 62.5 so)
            if (__any(top > mx[ct] + 8.f)) {
                const float m_new = fmaxf(mx[ct], top), down = __builtin_amdgcn_exp2f(mx[ct] - m_new);
                mx[ct] = m_new;
                sum[ct] *= down;
                if constexpr (!kWholeSum) total[ct] *= down;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[ct][i] *= down;
            }
            // Weights are exp2(s scale - mx) in one rounding, in which what the maximum lost in its own is a factor that cancels.
            // Beyond 2^28 that could be more than 2^16, and overflow further on: scores are rounded like the maximum there, so
            // that equal ones have equal weights, whatever their size.
            factor[ct] = a.scale_log2e;
            const bool far = fabsf(mx[ct]) > 0x1p28f && mx[ct] > kNoKey;
            if (__any(far)) {
                const float first = far ? a.scale_log2e : 1.f;   // (a column's own: its neighbours keep their rounding)
                factor[ct] = far ? 1.f : a.scale_log2e;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[ct][i] *= first;
            }
        }
        // keys behind the last (of the wave's last page): whatever lies there, their weights are zero and so are their values
        const bool clear = !more && j + kPageRows > hi;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 pf[CT][kP];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[ct][8 * h + e], factor[ct], -mx[ct]));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[ct][8 * h + e + 1], factor[ct], -mx[ct]));
                    if constexpr (kWholeSum) sum[ct] += p0 + p1;
                    unsigned w[kP];
                    if constexpr (PAIRED) {
                        split_pair<1>(p0, p1, w);
                        split_pair<1>(fmaf(__uint_as_float(w[0] << 16), second, p0), fmaf(__uint_as_float(w[0] & 0xffff0000u), second, p1), w);
                    } else split_pair<kP>(p0, p1, w);
#pragma unroll
                    for (int i = 0; i < kP; ++i) pf[ct][i][e / 2] = w[i];
                }
            if constexpr (!kWholeSum) {
                const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    total[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, pf[ct][0]), total[ct], 0, 0, 0);
            }
            float scale[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) scale[e] = exponent_scale((v_scale[2 * h + e / 4] >> (8 * (e % 4))) & 0xff);
            if (clear) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = 2 * h + e / 4, k = e % 4;
                    if (j + 16 * t + 4 * g4 + k < hi) continue;
                    scale[e] = 1.f;
#pragma unroll
                    for (int i = 0; i < BITS / 4; ++i) v_raw[t][(BITS / 4 * k + i) / 4][(BITS / 4 * k + i) % 4] = 0;
                }
            }
            // four columns of the lane's eight keys at a time
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                unsigned val[8][2];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = 2 * h + e / 4, k = e % 4;
                    if constexpr (BITS == 4) bf16_of4<BITS>(v_raw[t][0][k], part, scale[e], val[e]);
                    else bf16_of4<BITS>(v_raw[t][(2 * k + part) / 4][(2 * k + part) % 4], 0, scale[e], val[e]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u32x4 t;
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[e] = __builtin_amdgcn_perm(val[2 * e + 1][i / 2], val[2 * e][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                        for (int k = 0; k < kP; ++k)
                            acc[ct][4 * part + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t), __builtin_bit_cast(bf16x8, pf[ct][k]), acc[ct][4 * part + i], 0, 0, 0);
                }
            }
        }
        if constexpr (more) request_v(j + WAVES * kPageRows);
    };
    int j = lo + kPageRows * wave;
    if (j < hi) {
        request_k(j);
        request_v(j);
        for (; j + WAVES * kPageRows < hi; j += WAVES * kPageRows) weigh_page(j, std::true_type());
        weigh_page(j, std::false_type());
    }

    // the waves' results through LDS (register v of product i is column 8 (4 g4 + v) + i)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        if constexpr (!kWholeSum) sum[ct] = total[ct][0];
        else sum[ct] = wave_group_sum(sum[ct]);
        if (16 * ct + (PAIRED ? c16 % 8 : c16) < cols)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float* dst = &o_part[wave][16 * ct + c16][8 * (4 * g4 + v)];
                *reinterpret_cast<f32x4*>(dst) = f32x4{acc[ct][0][v], acc[ct][1][v], acc[ct][2][v], acc[ct][3][v]};
                *reinterpret_cast<f32x4*>(dst + 4) = f32x4{acc[ct][4][v], acc[ct][5][v], acc[ct][6][v], acc[ct][7][v]};
            }
        if (lane < 16) { stat[wave][16 * ct + lane][0] = mx[ct]; stat[wave][16 * ct + lane][1] = sum[ct]; }
    }
    __syncthreads();
    // From here on a wave takes whole columns, a lane two neighbouring values.
    float* const part0 = a.part + ((long long)bh * a.tiles + tile) * a.n_split * kCols * kPartStride;   // [slice][column]
    for (int q = wave; q < cols; q += WAVES) {
        float m_all = kNoKey, den = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m_all = fmaxf(m_all, stat[w][q][0]);
        Float2 v = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float wt = __builtin_amdgcn_exp2f(stat[w][q][0] - m_all);
            den = fmaf(stat[w][q][1], wt, den);
            Float2 x = {o_part[w][q][2 * lane], o_part[w][q][2 * lane + 1]};
            if constexpr (PAIRED) { x.x += o_part[w][q + 8][2 * lane]; x.y += o_part[w][q + 8][2 * lane + 1]; }
            v.x = fmaf(x.x, wt, v.x);
            v.y = fmaf(x.y, wt, v.y);
        }
        if (used == 1) {
            const bool some = sees(token(q)) > 0;
            store_pair(out_row(q) + 2 * lane, some ? v.x / den : 0.f, some ? v.y / den : 0.f);
        } else {
            float* const p = part0 + ((long long)sp * kCols + q) * kPartStride;
            put_shared(p + 2 * lane, v);
            if (lane == 0) put_shared(p + kHeadDim, Float2{m_all, den});
        }
    }
    if (used == 1) return;

    // the workgroup that draws the last ticket of its columns merges the slices
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) drawn = (int)(__hip_atomic_fetch_add(ticket, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 0xffff);
    __syncthreads();
    if (drawn != used - 1) return;
    // (a replayed graph calls by the same number again)
    if (threadIdx.x == 0) __hip_atomic_store(ticket, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (eight slices at a time: 32 at once 17.3 us for 8 tokens x 32 / 8 heads x 16000 keys, 14.8 so; several waves a column: even)
    constexpr int kBatch = 8;
    static_assert(kDecodeMaxSplit <= 64, "a lane weighs a slice");
    for (int q = wave; q < cols; q += WAVES) {
        const float* const p = part0 + q * kPartStride;
        // (the first slices' numerators are requested before their weights are known)
        Float2 x[kBatch];
        auto fetch = [&](int l) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) x[u] = get_shared(p + (long long)min(l + u, used - 1) * kCols * kPartStride + 2 * lane);
        };
        fetch(0);
        Float2 own = {kNoKey, 0.f};
        if (lane < used) own = get_shared(p + (long long)lane * kCols * kPartStride + kHeadDim);
        const float m_all = wave_group_max(row16_max(own.x));
        const float wt = lane < used ? __builtin_amdgcn_exp2f(own.x - m_all) : 0.f;   // of slice `lane`
        const float den = wave_group_sum(row16_sum(own.y * wt));
        Float2 num = {0.f, 0.f};
        for (int l = 0; l < used; l += kBatch) {
            if (l > 0) fetch(l);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wt), l + u));
                num.x = fmaf(x[u].x, w, num.x);
                num.y = fmaf(x[u].y, w, num.y);
            }
        }
        const bool some = sees(token(q)) > 0;
        store_pair(out_row(q) + 2 * lane, some ? num.x / den : 0.f, some ? num.y / den : 0.f);
    }
}

}  // namespace

size_t cache_bytes(int bits, long long caches, int capacity)
{
    const size_t pages = ((size_t)capacity + kPageRows - 1) / kPageRows;
    return (size_t)caches * pages * (bits == 4 ? page_bytes<4>() : page_bytes<8>());
}

CachePlan cache_plan(bool bf16, int B, int Hq, int Hkv, int n, int capacity, int n_cu)
{
    const long long cols = (long long)n * (Hq / Hkv), caches = (long long)B * Hkv;
    CachePlan p;
    // Two column tiles a workgroup halve the conversion of codes, where a workgroup for each compute unit is left (256
    // queries of 32 / 8 heads x 8192 keys: 73 us with one, 46 with two; with fewer: 8 x 5 tokens x 32 / 8 x 6000 20 -> 17,
    // but 4 x 8 x 4000 13.0 -> 15.1, 8 x 16000 14.6 -> 18.0, 128 x 2000 14.5 -> 16.2).
    p.col_tiles = bf16 && cols > 16 && caches * ((cols + 15) / 16) >= 2 * n_cu ? 2 : 1;
    p.tiles = (int)((cols + 16 * p.col_tiles - 1) / (16 * p.col_tiles));
    // Up to a workgroup of eight waves for each compute unit: of four waves two would leave twice the slices to merge
    // (bf16, 4 bits, 1 x 32 / 8 heads x 32768 keys 15.8 and 22.7 us with four, 8 x 32 / 8 x 8192 18.7 and 20.4, 8 x 32 / 32 x
    // 8192 53 and 56).  More than that, or where eight leave more than a quarter of the compute units out, of four:
    // their beginnings and ends overlap (64 x 32 / 8 x 2048 32.8 -> 29.7, 24 x 32 / 32 x up to 1000 24.0 -> 19.2; 4 x 40 / 40
    // x 12000 60.8 -> 52.5 in three slices, x 3000 even).
    const long long tiles = caches * p.tiles, of_8 = n_cu / tiles;
    p.waves = tiles > n_cu || 4 * tiles * of_8 <= 3 * n_cu ? 4 : 8;
    const long long most = std::min<long long>(kDecodeMaxSplit, ((long long)capacity + 255) / 256);
    p.split = tiles > n_cu ? 1 : (int)std::min(p.waves == 8 ? of_8 : 2 * n_cu / tiles, most);
    p.bytes = p.split == 1 ? 0 : (size_t)tiles * ((size_t)p.split * 16 * p.col_tiles * kPartStride + 2) * sizeof(float);
    return p;
}

size_t cache_scratch_bytes(int B, int Hq, int Hkv, int n)
{
    // (no plan for up to 256 compute units has more than 512 slices, and any only for up to 256 tiles of 16 columns)
    const long long tiles = (long long)B * Hkv * (((long long)n * (Hq / Hkv) + 15) / 16);
    if (tiles > 256) return 0;
    return (size_t)(std::min(512ll, kDecodeMaxSplit * tiles) * 16 * kPartStride + 2 * tiles) * sizeof(float);
}

static int pages_touched(int rows) { return (rows + kPageRows - 2) / kPageRows + 1; }   // by `rows` rows behind any others

bool cache_write_few(int Hkv, int m) { return 2ll * Hkv * m <= kAppendRows; }
long long cache_write_workgroups(int B, int Hkv, int m) { return cache_write_few(Hkv, m) ? B : 2ll * pages_touched(m) * B * Hkv; }
long long cache_read_workgroups(int B, int Hkv, int n) { return 2ll * pages_touched(n) * B * Hkv; }

hipError_t launch_cache_write(const CacheWriteArgs& in, int dtype, int bits, hipStream_t s)
{
    CacheWriteArgs a = in;
    a.pages = pages_touched(a.m);
    const bool few = cache_write_few(a.Hkv, a.m);
    const unsigned grid = (unsigned)cache_write_workgroups(a.B, a.Hkv, a.m);
#define TF_CACHE_WRITE(T, BITS)                                                                   \
    do {                                                                                          \
        if (few) cache_append_kernel<T, BITS><<<dim3(grid), dim3((unsigned)append_threads), 0, s>>>(a); \
        else cache_write_kernel<T, BITS><<<dim3(grid), dim3(256), 0, s>>>(a);                     \
    } while (0)
    const int append_threads = std::min(1024, (2 * a.Hkv * (few ? a.m : 1) * 16 + 63) / 64 * 64);
    if (dtype == 0) {
        if (bits == 4) TF_CACHE_WRITE(float, 4);
        else TF_CACHE_WRITE(float, 8);
    } else {
        if (bits == 4) TF_CACHE_WRITE(uint16_t, 4);
        else TF_CACHE_WRITE(uint16_t, 8);
    }
#undef TF_CACHE_WRITE
    const hipError_t e = hipGetLastError();
    if (few || e != hipSuccess) return e;
    cache_advance_kernel<<<dim3((unsigned)((a.B + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& in, int dtype, int bits, hipStream_t s)
{
    CacheReadArgs a = in;
    a.pages = pages_touched(a.n);
    const unsigned grid = (unsigned)cache_read_workgroups(a.B, a.Hkv, a.n);
    // (results that would push everything out of the 256 MB cache behind the L2s; smaller ones are what is used next)
    const bool stream = 2ll * (dtype == 0 ? 4 : 2) * kHeadDim * a.B * a.Hkv * a.n > (256ll << 20);
#define TF_CACHE_READ(T, BITS)                                                                    \
    do {                                                                                          \
        if (stream) cache_read_kernel<T, BITS, true><<<dim3(grid), dim3(256), 0, s>>>(a);         \
        else cache_read_kernel<T, BITS, false><<<dim3(grid), dim3(256), 0, s>>>(a);               \
    } while (0)
    if (dtype == 0) {
        if (bits == 4) TF_CACHE_READ(float, 4);
        else TF_CACHE_READ(float, 8);
    } else {
        if (bits == 4) TF_CACHE_READ(uint16_t, 4);
        else TF_CACHE_READ(uint16_t, 8);
    }
#undef TF_CACHE_READ
    return hipGetLastError();
}

hipError_t launch_cache_attend(const CacheAttendArgs& in, const CachePlan& plan, int dtype, int bits, hipStream_t s)
{
    CacheAttendArgs a = in;
    const long long tiles = (long long)a.B * a.Hkv * plan.tiles;
    a.tiles = plan.tiles; a.n_split = plan.split;
    a.by_ratio = divisor(a.Hq / a.Hkv); a.by_split = divisor(a.n_split); a.by_tiles = divisor(a.tiles); a.by_hkv = divisor(a.Hkv);
    a.tickets = (unsigned long long*)(a.part + tiles * a.n_split * 16 * plan.col_tiles * kPartStride);   // behind the partial results
    const unsigned grid = (unsigned)(tiles * a.n_split);
#define TF_CACHE_ATTEND(T, BITS, CT, PAIRED)                                                      \
    do {                                                                                          \
        if (plan.waves == 8) cache_attend_kernel<T, BITS, CT, 8, PAIRED><<<dim3(grid), dim3(512), 0, s>>>(a); \
        else cache_attend_kernel<T, BITS, CT, 4, PAIRED><<<dim3(grid), dim3(256), 0, s>>>(a);     \
    } while (0)
    const bool paired = (long long)a.n * (a.Hq / a.Hkv) <= 8;
    if (dtype == 0) {
        if (bits == 4) TF_CACHE_ATTEND(float, 4, 1, false);
        else TF_CACHE_ATTEND(float, 8, 1, false);
    } else if (plan.col_tiles == 2) {
        if (bits == 4) TF_CACHE_ATTEND(uint16_t, 4, 2, false);
        else TF_CACHE_ATTEND(uint16_t, 8, 2, false);
    } else if (paired) {
        if (bits == 4) TF_CACHE_ATTEND(uint16_t, 4, 1, true);
        else TF_CACHE_ATTEND(uint16_t, 8, 1, true);
    } else {
        if (bits == 4) TF_CACHE_ATTEND(uint16_t, 4, 1, false);
        else TF_CACHE_ATTEND(uint16_t, 8, 1, false);
    }
#undef TF_CACHE_ATTEND
    return hipGetLastError();
}

}  // namespace tf
