// Argument checks of the calls around a quantised cache, without a GPU: the host code of csrc/tokfilt_api.hip is compiled
// into this program (with AddressSanitizer and UndefinedBehaviorSanitizer on the host pass), a context is made by hand, and
// every refusal has to come before the device is asked for.  Exit status 0 = every call behaved as documented.
#include "../paper_2512_07090_amd/csrc/tokfilt_api.hip"

static int bad = 0;
static void expect(tf_ctx* c, tf_status got, tf_status want, const char* what)
{
    if (got != want || (want != TF_OK && c && !*tf_last_error(c))) { ++bad; printf("%s: status %d, not %d (%s)\n", what, got, want, c ? tf_last_error(c) : ""); }
    if (c) c->err[0] = 0;
}

static tf_params shape(int b, int hq, int hkv, int n, int dtype)
{
    tf_params p;
    memset(&p, 0, sizeof p);
    p.batch = b; p.n_q_heads = hq; p.n_kv_heads = hkv; p.seq = n; p.head_dim = 128; p.dtype = dtype;
    const long long q[3] = {(long long)hq * n * 128, n * 128ll, 128}, k[3] = {(long long)hkv * n * 128, n * 128ll, 128};
    for (int i = 0; i < 3; ++i) { p.q_stride[i] = p.o_stride[i] = q[i]; p.kv_stride[i] = k[i]; }
    return p;
}

int main()
{
    tf_ctx* c = new tf_ctx;
    memset(c, 0, sizeof *c);
    c->device = 0; c->n_cu = 256; c->n_xcd = 8;
    alignas(16) static unsigned char mem[4][256];
    void *K = mem[0], *V = mem[1], *Q = mem[2], *O = mem[3];
    alignas(16) static unsigned char ws[1 << 12];
    static int32_t len[4], four[64];
    const tf_status inv = TF_ERR_INVALID_ARG;
    tf_params p = shape(2, 8, 2, 4, TF_BF16);
    const tf_cache good = {K, V, len, nullptr, 64, TF_CACHE_FP4};

    // sizes: pages of 64 rows, whole ones
    if (tf_cache_bytes(&p, TF_CACHE_FP4, 1) != 4 * 4352 || tf_cache_bytes(&p, TF_CACHE_FP4, 64) != 4 * 4352 ||
        tf_cache_bytes(&p, TF_CACHE_FP4, 65) != 8 * 4352 || tf_cache_bytes(&p, TF_CACHE_FP8, 64) != 4 * 8448) { ++bad; printf("sizes\n"); }
    if (tf_cache_bytes(&p, 0, 64) || tf_cache_bytes(&p, 16, 64) || tf_cache_bytes(&p, 4, 0) || tf_cache_bytes(nullptr, 4, 64) ||
        tf_cache_workspace_bytes(nullptr)) { ++bad; printf("sizes of nothing\n"); }
    if (tf_cache_bytes(&p, TF_CACHE_FP8, 1 << 30) != 4ull * 16777216 * 8448) { ++bad; printf("large size\n"); }
    if (tf_cache_bytes(&p, TF_CACHE_FP8, (1 << 30) + 1) != 0) { ++bad; printf("size of too many rows\n"); }
    for (int b : {1, 3, 64}) for (int n : {1, 5, 300}) {
        const tf_params x = shape(b, 32, 8, n, TF_BF16);
        const size_t w = tf_cache_workspace_bytes(&x);
        if (w < 256 || w > (64u << 20)) { ++bad; printf("workspace\n"); }
    }
    // plans of the attention: every column in a tile, slices that a merge can hold, a workspace that is enough
    for (int dt = 0; dt < 2; ++dt) for (int b : {1, 2, 3, 5, 13, 40, 65, 300}) for (int hkv : {1, 2, 5, 8, 40}) for (int ratio : {1, 3, 4, 8, 17, 71})
        for (int n : {1, 2, 5, 16, 33, 257}) {
            const tf_params x = shape(b, hkv * ratio, hkv, n, dt);
            const size_t w = tf_cache_workspace_bytes(&x);
            for (int cap : {1, 64, 300, 5000, 1 << 30}) for (int cu = 1; cu <= 256; cu += cu < 8 ? 1 : 31) {
                const tf::CachePlan q = tf::cache_plan(dt != 0, b, hkv * ratio, hkv, n, cap, cu);
                const long long tiles = (long long)b * hkv * q.tiles;
                if (q.bytes > w || q.split < 1 || q.split > 64 || (q.waves != 4 && q.waves != 8) || (q.col_tiles != 1 && !(q.col_tiles == 2 && dt != 0)) ||
                    16ll * q.col_tiles * q.tiles < n * ratio || 16ll * q.col_tiles * (q.tiles - 1) >= n * ratio || (q.split > 1 && tiles * q.split > 2 * cu)) {
                    if (bad < 5) printf("plan of %d x %d / %d x %d, capacity %d, %d units\n", b, hkv * ratio, hkv, n, cap, cu);
                    ++bad;
                }
            }
        }
    // division by products
    for (unsigned by = 1; by < 70000; by += by < 300 ? 1 : 977) {
        const tf::Divisor d = tf::divisor(by);
        for (long long x : {0ll, (long long)by - 1, (long long)by, 5ll * by + 3, 0x7fffffffll, 0x7fffffffll / by * by, 0x7fffffffll / by * by - 1})
            if (x >= 0 && x <= 0x7fffffffll && ((((unsigned long long)x * d.mul >> 32) + (unsigned)x) >> d.shift) != (unsigned long long)x / by) { ++bad; printf("%lld / %u\n", x, by); }
    }
    { tf_params x = p; x.head_dim = 64; if (tf_cache_bytes(&x, 4, 64) || tf_cache_workspace_bytes(&x)) { ++bad; printf("shape\n"); } }

    auto write = [&](tf_ctx* cc, const tf_params* pp, const tf_cache* d, const void* k, const void* v, int m) { return tf_cache_write(cc, pp, d, k, v, nullptr, m, nullptr, nullptr); };
    expect(nullptr, write(nullptr, &p, &good, K, V, 4), inv, "write, no context");
    expect(c, write(c, nullptr, &good, K, V, 4), inv, "write, no parameters");
    expect(c, write(c, &p, nullptr, K, V, 4), inv, "write, no cache");
    for (int i = 0; i < 7; ++i) {
        tf_cache d = good;
        if (i == 0) d.k = nullptr;
        if (i == 1) d.v = nullptr;
        if (i == 2) d.len = nullptr;
        if (i == 3) d.capacity = 0;
        if (i == 4) d.format = 5;
        if (i == 5) d.k = (char*)K + 4;
        if (i == 6) d.v = (char*)V + 8;
        expect(c, write(c, &p, &d, K, V, 4), inv, "write, bad cache");
        expect(c, tf_cache_read(c, &p, &d, nullptr, K, V, nullptr), inv, "read, bad cache");
        expect(c, tf_cache_attend(c, &p, &d, Q, O, nullptr, ws, sizeof ws, nullptr), inv, "attend, bad cache");
    }
    expect(c, write(c, &p, &good, nullptr, V, 4), inv, "write, no K");
    expect(c, write(c, &p, &good, K, nullptr, 4), inv, "write, no V");
    expect(c, write(c, &p, &good, (char*)K + 2, V, 4), inv, "write, alignment");
    expect(c, write(c, &p, &good, K, V, 0), inv, "write, m = 0");
    expect(c, write(c, &p, &good, K, V, 5), inv, "write, m > seq");
    { tf_cache d = good; d.capacity = (1 << 30) + 1; expect(c, write(c, &p, &d, K, V, 4), TF_ERR_UNSUPPORTED, "write, too many rows of a cache"); }
    { tf_cache d = good; d.capacity = 1 << 30; tf_params x = shape(65535, 128, 128, 1, TF_F32);
      expect(c, write(c, &x, &d, K, V, 1), TF_ERR_UNSUPPORTED, "write, too large a cache"); }
    { tf_params x = shape(128, 128, 128, 1 << 23, TF_F32);
      expect(c, write(c, &x, &good, K, V, 1 << 23), TF_ERR_UNSUPPORTED, "write, too many rows");
      expect(c, tf_cache_read(c, &x, &good, nullptr, K, V, nullptr), TF_ERR_UNSUPPORTED, "read, too many rows"); }
    expect(c, tf_cache_read(c, &p, &good, nullptr, nullptr, V, nullptr), inv, "read, no K");
    { tf_params x = p; x.kv_stride[0] = 0; expect(c, tf_cache_read(c, &x, &good, nullptr, K, V, nullptr), inv, "read, folded"); }
    auto attend = [&](const tf_params* pp, const void* q, void* o, void* w, size_t n) { return tf_cache_attend(c, pp, &good, q, o, nullptr, w, n, nullptr); };
    expect(c, attend(&p, nullptr, O, ws, sizeof ws), inv, "attend, no Q");
    expect(c, attend(&p, Q, nullptr, ws, sizeof ws), inv, "attend, no O");
    expect(c, attend(&p, Q, Q, ws, sizeof ws), inv, "attend, in place");
    expect(c, attend(&p, Q, O, nullptr, 0), inv, "attend, no workspace");
    expect(c, attend(&p, Q, O, ws + 1, sizeof ws - 1), inv, "attend, workspace alignment");
    { tf_cache d = good; d.capacity = 5000;
      expect(c, tf_cache_attend(c, &p, &d, Q, O, nullptr, ws, 16, nullptr), TF_ERR_WORKSPACE_TOO_SMALL, "attend, small workspace"); }
    { tf_params x = p; x.o_stride[1] = 0; expect(c, attend(&x, Q, O, ws, sizeof ws), inv, "attend, folded"); }
    { tf_params x = shape(1024, 128, 1, 1 << 19, TF_F32); expect(c, attend(&x, Q, O, ws, sizeof ws), TF_ERR_UNSUPPORTED, "attend, too many queries"); }

    tf_decode_state st = {(double*)K, (double*)V, four, four, (float*)four, four, four, K, V, 64, 0};
    for (int f : {0, 3, 16, -4}) {
        expect(c, tf_decode_step_q(c, &p, 0.f, &st, f, Q, K, V, O, (uint8_t*)four, (float*)four, ws, sizeof ws, nullptr), inv, "step, format");
        expect(c, tf_decode_prefill_q(c, &p, 0.f, 0.f, &st, f, Q, K, V, (uint8_t*)four, four, four, (float*)four, O, ws, sizeof ws, nullptr), inv, "prefill, format");
    }
    { tf_decode_state big = st; big.capacity = (1 << 30) + 1;
      expect(c, tf_decode_step_q(c, &p, 0.f, &big, 4, Q, K, V, O, (uint8_t*)four, (float*)four, ws, sizeof ws, nullptr), TF_ERR_UNSUPPORTED, "step, too many rows"); }
    expect(nullptr, tf_decode_step_q(nullptr, &p, 0.f, &st, 4, Q, K, V, O, (uint8_t*)four, (float*)four, ws, sizeof ws, nullptr), inv, "step, no context");
    expect(nullptr, tf_decode_prefill_q(nullptr, &p, 0.f, 0.f, &st, 4, Q, K, V, (uint8_t*)four, four, four, (float*)four, O, ws, sizeof ws, nullptr), inv, "prefill, no context");

    tf_rotary r;
    memset(&r, 0, sizeof r);
    r.freq = (const double*)K; r.eps = 1e-6f; r.rot_dim = 128;
    auto rotate = [&](const tf_rotary* rr, const tf_params* pp, const void* q, const void* k, void* qo, void* ko) { return tf_norm_rotate(c, pp, rr, q, k, qo, ko, nullptr); };
    expect(nullptr, tf_norm_rotate(nullptr, &p, &r, Q, K, O, V, nullptr), inv, "rotate, no context");
    expect(c, rotate(nullptr, &p, Q, K, O, V), inv, "rotate, no description");
    for (int i = 0; i < 12; ++i) {
        tf_rotary x = r;
        if (i == 0) x.rot_dim = 8;
        if (i == 1) x.rot_dim = 144;
        if (i == 2) x.rot_dim = -16;
        if (i == 3) x.freq = nullptr;
        if (i == 4) x.eps = 0.f;
        if (i == 5) x.eps = NAN;
        if (i == 6) x.eps = INFINITY;
        if (i == 7) x.interleaved = 2;
        if (i == 8) x.reserved = 1;
        if (i == 9) x.q_weight = (const float*)K + 1;
        if (i == 10) x.k_weight = (const float*)K + 2;
        if (i == 11) x.freq = (const double*)((const float*)K + 1);
        expect(c, rotate(&x, &p, Q, K, O, V), inv, "rotate, bad description");
    }
    expect(c, rotate(&r, &p, nullptr, nullptr, nullptr, nullptr), inv, "rotate, nothing");
    expect(c, rotate(&r, &p, Q, K, nullptr, V), inv, "rotate, no output");
    expect(c, rotate(&r, &p, Q, nullptr, O, V), inv, "rotate, no input");
    expect(c, rotate(&r, &p, (char*)Q + 2, K, O, V), inv, "rotate, alignment");
    { tf_params x = shape(1024, 65535, 1, 1 << 20, TF_F32); expect(c, rotate(&r, &x, Q, K, O, V), TF_ERR_UNSUPPORTED, "rotate, too many rows"); }
    { tf_params x = p; x.o_stride[0] *= 2; expect(c, rotate(&r, &x, Q, K, Q, V), inv, "rotate, in place elsewhere"); }
    { tf_params x = p; x.kv_stride[0] = 0; expect(c, rotate(&r, &x, Q, K, O, V), inv, "rotate, folded"); }

    delete c;
    printf("cache refusals: %d failures\n", bad);
    return bad ? 1 : 0;
}
