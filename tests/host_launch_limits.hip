// Shapes whose launch would have 2^32 threads or more are refused as unsupported before the device is asked for, and shapes
// right below that are not.  No GPU: the host code of csrc/tokfilt_api.hip is compiled into this program, and its context
// names a device that no machine has, so a call that is not refused ends where it would choose the device.
#include "../paper_2512_07090_amd/csrc/tokfilt_api.hip"

static int bad = 0;
static void expect(tf_ctx* c, tf_status got, bool refused, const char* what)
{
    const tf_status want = refused ? TF_ERR_UNSUPPORTED : TF_ERR_DEVICE;
    if (got != want || !*tf_last_error(c)) { ++bad; printf("%s: status %d, not %d (%s)\n", what, got, want, tf_last_error(c)); }
    c->err[0] = 0;
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
    c->device = 1 << 20; c->n_cu = 256; c->n_xcd = 8;
    alignas(16) static unsigned char mem[4][256];
    void *K = mem[0], *V = mem[1], *Q = mem[2], *O = mem[3];
    alignas(16) static unsigned char ws[1 << 12];
    static int32_t len[4];

    // norm and rotation: workgroups of 256 threads for 16 heads of up to four tokens of a tensor
    tf_rotary r;
    memset(&r, 0, sizeof r);
    r.freq = (const double*)K; r.eps = 1e-6f; r.rot_dim = 128;
    auto rotate = [&](int b, int hq, int hkv, int n, bool with_q, bool with_k) {
        const tf_params p = shape(b, hq, hkv, n, TF_F32);
        return tf_norm_rotate(c, &p, &r, with_q ? Q : nullptr, with_k ? K : nullptr, with_q ? O : nullptr, with_k ? V : nullptr, nullptr);
    };
    expect(c, rotate(1, 1, 1, 1 << 25, true, true), true, "rotate, 2^24 workgroups");
    expect(c, rotate(1, 1, 1, (1 << 25) - 4, true, true), false, "rotate, 2^24 - 2 workgroups");
    expect(c, rotate(1, 1, 1, (1 << 25) - 3, true, true), true, "rotate, a last token alone");
    expect(c, rotate(1, 1, 1, (1 << 26) - 4, true, false), false, "rotate, queries alone");
    expect(c, rotate(1, 1, 1, 1 << 26, false, true), true, "rotate, keys alone");
    expect(c, rotate(1, 32, 16, 22369616, true, true), false, "rotate, three workgroups a token");
    expect(c, rotate(1, 32, 16, 22369624, true, true), true, "rotate, three workgroups a token, too many");
    expect(c, rotate(65535, 1, 1, 3, true, true), false, "rotate, three tokens a row");
    expect(c, rotate(65535, 1344, 1, 3, true, true), false, "rotate, three tokens a row, 85 workgroups each");
    expect(c, rotate(65535, 1345, 1, 3, true, true), true, "rotate, three tokens a row, 86 workgroups each");

    // a cache: 256 threads for each page of each tensor that rows touch; few new rows in one workgroup for a batch row
    const tf_cache cache = {K, V, len, nullptr, 64, TF_CACHE_FP4};
    auto write = [&](int b, int hkv, int m) { const tf_params p = shape(b, hkv, hkv, m, TF_F32); return tf_cache_write(c, &p, &cache, K, V, nullptr, m, nullptr, nullptr); };
    auto read = [&](int b, int hkv, int n) { const tf_params p = shape(b, hkv, hkv, n, TF_F32); return tf_cache_read(c, &p, &cache, nullptr, K, V, nullptr); };
    expect(c, write(65535, 128, 1), false, "write, one row each");
    expect(c, write(65535, 128, 5), true, "write, five rows each");
    expect(c, write(32767, 128, 5), false, "write, five rows each of half as many");
    expect(c, read(65535, 128, 1), false, "read, one row each");
    expect(c, read(65535, 128, 2), true, "read, two rows each");

    // attention: 256 threads for 16 columns of a cache where there are that many
    auto attend = [&](int b, int hkv, int n) { const tf_params p = shape(b, hkv, hkv, n, TF_F32); return tf_cache_attend(c, &p, &cache, Q, O, nullptr, ws, sizeof ws, nullptr); };
    expect(c, attend(65535, 128, 32), false, "attend, two tiles a cache");
    expect(c, attend(65535, 128, 33), true, "attend, three tiles a cache");
    { const tf_params p = shape(65535, 128, 128, 33, TF_BF16);   // (tiles of 32 columns)
      expect(c, tf_cache_attend(c, &p, &cache, Q, O, nullptr, ws, sizeof ws, nullptr), false, "attend, two double tiles a cache"); }

    delete c;
    printf("launch limits: %d failures\n", bad);
    return bad ? 1 : 0;
}
