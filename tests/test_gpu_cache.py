"""The cache in 4 and 8 bits through the C ABI: what is written byte for byte, what is read back exactly, attention over it
against 64 bits on what the codes stand for, and the per-token path on it against the same path on whole rows.

Tolerance of the attention, with A = sum of weight |v| and S = the largest scale * sum |q k| of a query and one of its keys:
codes are exact, so a score is off by the fp32 rounding of 128 products (2^-24 each, some 16 additions deep on the matrix
pipe: 2^-20 S), of its scaling and of the exponent (2^-22 S); a weight by as much and, for bf16 queries, by the rounding of
its two bf16 parts (2^-16); sums over up to some hundred steps add 2^-18.  Both the numerator and the denominator carry that:
  fp32  |o - ref| <= (2^-18 S + 2^-17) A
  bf16  |o - ref| <= (2^-18 S + 2^-15) A + 2^-8 |ref|   (the output's own rounding)
A call with many queries rounds a weight to bf16 once (|d| <= 2^-8), numerator and denominator alike, so that the result is
sum w (1 + d) v / sum w (1 + d), off by at most 2^-8 / (1 - 2^-8) (A + |ref|) < (2^-8 + 2^-15) (A + |ref|):
  bf16  |o - ref| <= (2^-18 S + 2^-8 + 2^-14) (A + |ref|) + 2^-8 |ref|
"""
import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_2512_07090_amd import binding as B
from paper_2512_07090_amd import synth

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c = B.Context(0)
    yield c
    c.close()


def _say(msg):
    print("[case] " + msg, flush=True)


def _params(dt, Bn, Hq, Hkv, n, **kw):
    return B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), DT[dt], 0.0, **kw)


def _rows(shape, dt, seed, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    return (x * torch.exp(spread * torch.randn(shape[-1], generator=g, device="cuda"))).to(DT[dt])


def _hard(x):
    """Some rows that are hard to round: zeros, one value, borders between codes, far ends of the range, tiny ones."""
    x = x.clone()
    flat = x.view(-1, 128)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device=x.device)
    rows = [torch.zeros(128, device=x.device), torch.full((128,), -3.5, device=x.device), ties.repeat(16),
            -ties.repeat(16) * 2.0 ** 80, ties.repeat(16) * 2.0 ** -120, torch.full((128,), 2.0 ** 125, device=x.device),
            torch.full((128,), 2.0 ** -130, device=x.device), torch.arange(128, device=x.device) * 1.0,
            448.0 * (1 + torch.arange(128, device=x.device) / 64.0), torch.exp2(-torch.arange(128, device=x.device) / 6.0)]
    for i, r in enumerate(rows):
        flat[(i * 7) % flat.shape[0]] = r.to(x.dtype)
    return x


def _blob(t, Bn, Hkv, bits):
    return t.cpu().numpy().reshape(Bn, Hkv, -1, ref.page_bytes(bits))


def _f64(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("case", [   # dtype, bits, batch, KV heads, n, rows held before (per batch row), capacity
    ("bf16", 4, 1, 1, 1, [0], 1), ("bf16", 4, 2, 3, 130, [0, 61], 200), ("bf16", 8, 2, 2, 64, [64, 1], 128),
    ("f32", 4, 3, 2, 77, [3, 0, 500], 577), ("f32", 8, 1, 5, 200, [63], 300), ("bf16", 8, 4, 8, 1, [0, 1, 63, 64], 65),
    ("bf16", 4, 2, 128, 5, [15, 16], 40)])
def test_write_makes_the_pages_and_leaves_the_rest(ctx, case):
    dt, bits, Bn, Hkv, n, held, cap = case
    _say("cache write %s" % (case,))
    p = _params(dt, Bn, Hkv, Hkv, n)
    k, v = (_hard(_rows((Bn, Hkv, n, 128), dt, s)) for s in (1, 2))
    c = B.QuantCache(p, cap, bits)
    c.k.fill_(0xA5)
    c.v.fill_(0x5A)
    c.len.copy_(torch.tensor(held, dtype=torch.int32))
    ctx.tf_cache_write(p, c.desc, k, v, None, n, None)
    torch.cuda.synchronize()
    assert c.len.tolist() == [min(h + n, cap) for h in held]
    assert c.overflow.tolist() == [int(h + n > cap) for h in held]
    for t, x, is_value, fill in ((c.k, k, False, 0xA5), (c.v, v, True, 0x5A)):
        want = np.full((Bn, Hkv, (cap + 63) // 64, ref.page_bytes(bits)), fill, np.uint8)
        at, se = ref.places(bits, is_value)
        code, ex = ref.quantise(_f64(x), bits)
        for b, h in enumerate(held):
            for i in range(min(n, cap - h)):
                page, r = (h + i) // 64, (h + i) % 64
                if bits == 4:
                    want[b, :, page, at[r, 0::2]] = (code[b, :, i, 0::2] | code[b, :, i, 1::2] << 4).T
                else:
                    want[b, :, page, at[r]] = code[b, :, i].T
                want[b, :, page, se[r]] = ex[b, :, i].T
        np.testing.assert_array_equal(_blob(t, Bn, Hkv, bits), want)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_write_kept_rows_in_parts_and_read_back(ctx, dt, bits):
    """Kept positions, ragged counts (0 among them), strided storage, two calls in a row; read back from anywhere."""
    Bn, Hkv, n, cap = 3, 4, 150, 260
    _say("cache write kept %s %d" % (dt, bits))
    k, v = (_hard(_rows((Bn, n, Hkv, 128), dt, s)).transpose(1, 2) for s in (3, 4))
    p = _params(dt, Bn, Hkv, Hkv, n, kv_stride=k.stride()[:3])
    c = B.QuantCache(p, cap, bits)
    c.k.fill_(0xFF)
    c.v.fill_(0xFF)
    g = torch.Generator().manual_seed(5)
    held = [0] * Bn
    want = [[], []]
    for counts in ([150, 0, 71], [1, 33, 150]):
        m = 150
        idx = torch.full((Bn, m), -1, dtype=torch.int32)
        for b, cnt in enumerate(counts):
            idx[b, :cnt] = torch.randperm(n, generator=g)[:cnt].sort().values.int()
        ctx.tf_cache_write(p, c.desc, k, v, idx.cuda(), m, torch.tensor(counts, dtype=torch.int32).cuda())
        for w, x in zip(want, (k, v)):
            w.append([x[b][:, idx[b, :cnt].long().cuda()] for b, cnt in enumerate(counts)])
        held = [h + cnt for h, cnt in zip(held, counts)]
    torch.cuda.synchronize()
    assert c.len.tolist() == held and c.overflow.tolist() == [0] * Bn
    for start in (None, [0, 10, 149], [150, 33, 221], [-3, 300, 64]):
        out = [torch.full_like(k.contiguous(), 77.0) for _ in range(2)]
        p2 = _params(dt, Bn, Hkv, Hkv, n)
        ctx.tf_cache_read(p2, c.desc, None if start is None else torch.tensor(start, dtype=torch.int32).cuda(), *out)
        torch.cuda.synchronize()
        for o, w in zip(out, want):
            for b in range(Bn):
                rows = torch.cat([part[b] for part in w], 1)
                s = max(0, start[b]) if start else 0
                rows = rows[:, s:s + n]
                np.testing.assert_array_equal(_f64(o[b, :, :rows.shape[1]]), ref.values(*ref.quantise(_f64(rows), bits), bits))
                assert (o[b, :, rows.shape[1]:] == 77.0).all()


def _quant_cache(p, dt, bits, Bn, Hkv, lens, cap, seed):
    """A cache of `lens` rows (all else 0xFF: NaN codes and scales in 8 bits) and what it stands for."""
    k, v = (_rows((Bn, Hkv, cap, 128), "f32", seed + i, 0.4) for i in range(2))
    c = B.QuantCache(p, cap, bits)
    out = []
    for x, t, is_value in ((k, c.k, False), (v, c.v, True)):
        code, ex = ref.quantise(_f64(x), bits)
        blob = ref.pack(code, ex, bits, is_value)
        at, se = ref.places(bits, is_value)
        for b, m in enumerate(lens):
            for row in range(m, blob.shape[2] * 64):
                blob[b, :, row // 64, at[row % 64]] = 0xFF
                blob[b, :, row // 64, se[row % 64]] = 0xFF
        t.copy_(torch.from_numpy(blob).reshape(-1))
        out.append(torch.from_numpy(ref.values(code, ex, bits)).cuda())
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return c, out[0], out[1]


def _check_attention(o, want, dt, many=False):
    r, A, S = want
    err = (o.double() - r).abs()
    if many:
        tol = (2.0 ** -18 * S + 2.0 ** -8 + 2.0 ** -14) * (A + r.abs()) + 2.0 ** -8 * r.abs()
        assert (err <= tol).all(), (err - tol).max().item()
        return
    tol = (2.0 ** -18 * S + (2.0 ** -17 if dt == "f32" else 2.0 ** -15)) * A + (2.0 ** -8 * r.abs() if dt == "bf16" else 0)
    assert (err <= tol).all(), (err - tol).max().item()


@pytest.mark.parametrize("case", [   # dtype, bits, batch, query heads, KV heads, new tokens, lengths, counts, capacity
    ("bf16", 4, 1, 1, 1, 1, [1], None, 1), ("bf16", 4, 4, 8, 2, 1, [0, 1, 63, 64], None, 70),
    ("bf16", 4, 3, 4, 4, 1, [65, 127, 128], None, 1000), ("bf16", 4, 2, 32, 8, 1, [1000, 3001], None, 3100),
    ("bf16", 8, 2, 10, 2, 1, [2049, 500], None, 2049), ("f32", 4, 2, 6, 2, 1, [129, 900], None, 900),
    ("f32", 8, 3, 4, 4, 1, [64, 0, 701], None, 777), ("bf16", 4, 1, 71, 1, 1, [333], None, 400),
    ("bf16", 8, 1, 128, 8, 1, [200], None, 200), ("bf16", 4, 2, 8, 2, 7, [7, 300], None, 320),
    ("bf16", 4, 3, 4, 2, 33, [33, 200, 20], [33, 10, 0], 256), ("bf16", 8, 2, 6, 2, 20, [5, 400], [20, 19], 401),
    ("f32", 4, 2, 4, 1, 9, [100, 9], [9, 4], 128), ("f32", 8, 1, 4, 4, 40, [130], None, 130),
    ("bf16", 4, 1, 8, 8, 100, [1500], None, 1600), ("bf16", 4, 2, 8, 1, 64, [64, 700], [1, 64], 700),
    ("bf16", 8, 9, 8, 1, 20, [20 + 70 * b for b in range(9)], None, 600),
    # more columns than compute units: four waves a workgroup, two column tiles where a cache has many of them
    ("bf16", 4, 40, 8, 8, 1, [17 * b for b in range(40)], None, 700), ("f32", 8, 40, 8, 8, 1, [5 * b + 1 for b in range(40)], None, 200),
    ("bf16", 8, 4, 40, 40, 1, [1300, 1, 700, 65], None, 1300), ("f32", 4, 4, 40, 40, 1, [1025, 64, 0, 513], None, 1100),
    ("bf16", 4, 2, 32, 8, 130, [200, 140], [130, 77], 256), ("bf16", 8, 16, 8, 8, 70, [70 + 29 * b for b in range(16)], None, 530),
    ("bf16", 4, 9, 24, 8, 40, [40 * b for b in range(9)], [40 - 4 * b for b in range(9)], 330),
    ("bf16", 8, 1, 64, 4, 300, [290], None, 300)])
def test_attend_matches_64_bits(ctx, case):
    dt, bits, Bn, Hq, Hkv, n, lens, counts, cap = case
    _say("cache attend %s" % (case,))
    p = _params(dt, Bn, Hq, Hkv, n)
    c, k, v = _quant_cache(p, dt, bits, Bn, Hkv, lens, cap, 20)
    q = _rows((Bn, Hq, n, 128), dt, 9, 0.2)
    o = torch.full_like(q, float("nan"))
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    ctx.tf_cache_attend(p, c.desc, q, o, cnt, ws)
    torch.cuda.synchronize()
    # a call whose columns (queries x heads of a KV head) are many tiles of 16
    many = dt == "bf16" and n * (Hq // Hkv) > 16 and Bn * Hkv * -(-n * (Hq // Hkv) // 16) >= 512
    _check_attention(o, ref.attend(q.double(), k, v, lens, counts or [n] * Bn, 128 ** -0.5), dt, many)


def test_attend_strided_scaled_and_sharp(ctx):
    """Token-major storage, a scale of its own, and queries large enough that one key takes nearly all of the weight."""
    Bn, Hq, Hkv, n, cap = 2, 8, 2, 3, 700
    _say("cache attend strided")
    c, k, v = _quant_cache(_params("bf16", Bn, Hq, Hkv, n), "bf16", 4, Bn, Hkv, [700, 650], cap, 30)
    q = (_rows((Bn, n, Hq, 128), "bf16", 31, 0.2) * 8).transpose(1, 2)
    o = torch.full((Bn, n, Hq, 136), float("nan"), dtype=torch.bfloat16, device="cuda")[..., :128].transpose(1, 2)
    p = _params("bf16", Bn, Hq, Hkv, n, q_stride=q.stride()[:3], o_stride=o.stride()[:3], softmax_scale=0.11)
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
    torch.cuda.synchronize()
    _check_attention(o, ref.attend(q.double(), k, v, [700, 650], [n] * Bn, float(np.float32(0.11))), "bf16")
    assert torch.isnan(o.as_strided((Bn, n, Hq, 8), (n * Hq * 136, Hq * 136, 136, 1), o.storage_offset() + 128)).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_on_both_sides_of_the_slices_borders(ctx, dt):
    """Lengths at which a row's slices change in size, and their number."""
    lens, cap = [513, 4097, 8193, 1025, 2049], 8200
    Bn, Hq, Hkv = len(lens), 4, 1
    _say("cache attend slices %s" % dt)
    p = _params(dt, Bn, Hq, Hkv, 1)
    c, k, v = _quant_cache(p, dt, 4, Bn, Hkv, lens, cap, 36)
    q = _rows((Bn, Hq, 1, 128), dt, 37, 0.2)
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    for less in (0, 1, 2, 65, 513):
        cur = [n - less for n in lens]
        c.len.copy_(torch.tensor(cur, dtype=torch.int32))
        o = torch.full_like(q, float("nan"))
        ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
        torch.cuda.synchronize()
        _check_attention(o, ref.attend(q.double(), k, v, cur, [1] * Bn, 128 ** -0.5), dt)


@pytest.mark.parametrize("case", [("bf16", 2, 8, 2, 3), ("bf16", 2, 8, 2, 12), ("f32", 2, 4, 2, 5), ("bf16", 20, 16, 8, 40)])
def test_padding_may_hold_anything(ctx, case):
    """Queries from count on, and rows of the cache behind its length, are NaN and infinities: no trace of them."""
    dt, Bn, Hq, Hkv, n = case
    _say("cache attend padding %s" % (case,))
    lens, counts = [200 + 13 * b for b in range(Bn)], [n - 1 - b % (n - 1) for b in range(Bn)]
    p = _params(dt, Bn, Hq, Hkv, n)
    c, k, v = _quant_cache(p, dt, 8, Bn, Hkv, lens, 520, 33)
    q = _rows((Bn, Hq, n, 128), dt, 34, 0.2)
    clean = q.clone()
    for b in range(Bn):
        q[b, :, counts[b]:] = float("nan") if b % 2 else float("inf")
    cnt = torch.tensor(counts, dtype=torch.int32, device="cuda")
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    outs = []
    for x in (q, clean):
        o = torch.full_like(q, float("nan"))
        ctx.tf_cache_attend(p, c.desc, x, o, cnt, ws)
        outs.append(o)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    for b in range(Bn):
        assert not outs[0][b, :, counts[b]:].any()
    assert torch.isfinite(outs[0].float()).all()


def test_attend_row_does_not_depend_on_its_neighbours(ctx):
    Bn, Hq, Hkv, n, cap = 5, 8, 2, 4, 1500
    _say("cache attend neighbours")
    p = _params("bf16", Bn, Hq, Hkv, n)
    lens = [1500, 900, 64, 1100, 5]
    c, k, v = _quant_cache(p, "bf16", 4, Bn, Hkv, lens, cap, 40)
    q = _rows((Bn, Hq, n, 128), "bf16", 41)
    ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    first = None
    for others in (lens, [0] * Bn, [1500] * Bn):
        for b in range(Bn):
            cur = list(others)
            cur[b] = lens[b]
            c.len.copy_(torch.tensor(cur, dtype=torch.int32))
            # (rows behind a row's own length hold NaN codes: only lengths that are there are compared)
            o = torch.empty_like(q)
            ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
            if first is None:
                first = o.clone()
            assert torch.equal(o[b], first[b]), (others, b)


def test_calls_on_two_streams_and_from_replayed_graphs(ctx):
    """A token as it is served (append, attend) captured once and replayed: every replay appends another token.  Another
    stream works on a cache of its own with a workspace of its own at the same time."""
    Bn, Hq, Hkv, cap = 2, 8, 2, 600
    _say("cache graph")
    p = _params("bf16", Bn, Hq, Hkv, 1)
    p0 = _params("bf16", Bn, Hq, Hkv, 500)
    k0, v0 = (_rows((Bn, Hkv, 500, 128), "bf16", s) for s in (50, 51))
    steps = [[_rows((Bn, h, 1, 128), "bf16", 60 + 3 * i + j) for j, h in enumerate((Hq, Hkv, Hkv))] for i in range(6)]

    def eager():
        c = B.QuantCache(p, cap, 4)
        ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        ctx.tf_cache_write(p0, c.desc, k0, v0, None, 500, None)
        outs = []
        for q, k, v in steps:
            o = torch.empty_like(q)
            ctx.tf_cache_write(p, c.desc, k, v, None, 1, None)
            ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
            outs.append(o)
        torch.cuda.synchronize()
        return outs, c
    want, cw = eager()

    c = B.QuantCache(p, cap, 4)
    ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.empty_like(t) for t in steps[0])
    o = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ctx.tf_cache_write(p0, c.desc, k0, v0, None, 500, None)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ctx.tf_cache_write(p, c.desc, k, v, None, 1, None)
        ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
    other = B.QuantCache(p, cap, 4)
    ws2 = torch.empty_like(ws)
    o2 = torch.empty_like(q)
    s2 = torch.cuda.Stream()
    s2.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s2):
        ctx.tf_cache_write(p0, other.desc, k0, v0, None, 500, None)
    for i, (a, b, d) in enumerate(steps):
        q.copy_(a)
        k.copy_(b)
        v.copy_(d)
        torch.cuda.synchronize()
        with torch.cuda.stream(s2):
            ctx.tf_cache_write(p, other.desc, b, d, None, 1, None)
            ctx.tf_cache_attend(p, other.desc, a, o2, None, ws2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[i]) and torch.equal(o2, want[i]), i
        assert c.len.tolist() == [501 + i] * Bn
    assert torch.equal(c.len, cw.len)


def test_rows_beyond_4_gib(ctx):
    """Caches of more than 2^32 bytes: rows appended at the end of every head's, read back, and attended to among 2^24 - 1
    others of zeros, whose scores are 0 and whose values add nothing."""
    Hkv, ratio, cap, n = 4, 2, 1 << 24, 37
    _say("cache beyond 4 GiB")
    p = _params("bf16", 1, Hkv * ratio, Hkv, n)
    assert B.tf_cache_bytes(p, 4, cap) > 1 << 32
    c = B.QuantCache(p, cap, 4)
    c.k.zero_()
    c.v.zero_()
    c.len.fill_(cap - n)
    k, v = (_rows((1, Hkv, n, 128), "bf16", s, 0.2) for s in (90, 91))
    ctx.tf_cache_write(p, c.desc, k, v, None, n, None)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    ctx.tf_cache_read(p, c.desc, torch.tensor([cap - n], dtype=torch.int32, device="cuda"), ko, vo)
    torch.cuda.synchronize()
    assert c.len.item() == cap and c.overflow.item() == 0
    kk, vv = (torch.from_numpy(ref.values(*ref.quantise(_f64(x), 4), 4)).cuda() for x in (k, v))
    assert torch.equal(ko.double(), kk) and torch.equal(vo.double(), vv)
    one = _params("bf16", 1, Hkv * ratio, Hkv, 1)
    q = (4 * kk[:, :, -1:].repeat_interleave(ratio, 1)).bfloat16()       # far from all but its own key
    o = torch.full_like(q, float("nan"))
    ctx.tf_cache_attend(one, c.desc, q, o, None, torch.empty(B.tf_cache_workspace_bytes(one), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for h in range(Hkv * ratio):
        s = (kk[0, h // ratio] @ q[0, h, 0].double()) * 128 ** -0.5
        top = s.max().clamp(min=0.0)
        w = torch.exp(s - top)
        den = w.sum() + (cap - n) * torch.exp(-top)
        out, A = (w[:, None] * vv[0, h // ratio]).sum(0) / den, (w[:, None] * vv[0, h // ratio].abs()).sum(0) / den
        S = (kk[0, h // ratio].abs() @ q[0, h, 0].double().abs()).max() * 128 ** -0.5
        # the denominator's 2^24 / 64 / 8 / 64 additions a lane of equal terms are exact to 2^-24 each
        assert ((o[0, h, 0].double() - out).abs() <= (2.0 ** -18 * S + 2.0 ** -14) * A + 2.0 ** -8 * out.abs()).all(), h


def test_the_same_call_gives_the_same_bits(ctx):
    Bn, Hq, Hkv, cap = 3, 16, 4, 5000
    _say("cache attend repeated")
    for n in (1, 6):
        p = _params("bf16", Bn, Hq, Hkv, n)
        c, _, _ = _quant_cache(p, "bf16", 4, Bn, Hkv, [5000, 4321, 700], cap, 95)
        q = _rows((Bn, Hq, n, 128), "bf16", 96)
        ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        outs = [torch.empty_like(q) for _ in range(12)]
        for o in outs:
            ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(o, outs[0]) for o in outs)


def test_two_graphs_share_a_workspace(ctx):
    """Two layers captured apart, with other lengths and other numbers of slices, replayed in turn over one workspace."""
    Bn, Hq, Hkv, cap = 2, 8, 2, 3000
    _say("cache two graphs")
    layers, graphs, s = [], [], torch.cuda.Stream()
    ws = None
    for n, lens in ((1, [2900, 40]), (5, [700, 3000])):
        p = _params("bf16", Bn, Hq, Hkv, n)
        c, k, v = _quant_cache(p, "bf16", 4, Bn, Hkv, lens, cap, 70 + n)
        q = _rows((Bn, Hq, n, 128), "bf16", 80 + n)
        o, want = torch.empty_like(q), torch.empty_like(q)
        ws = torch.full((2 * B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws
        assert ws.numel() >= B.tf_cache_workspace_bytes(p)
        ctx.tf_cache_attend(p, c.desc, q, want, None, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
        layers.append((o, want, c, q))
        graphs.append(g)
    for turn in (0, 1, 0, 0, 1, 1, 0):
        layers[turn][0].fill_(float("nan"))
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert torch.equal(layers[turn][0], layers[turn][1]), turn


@pytest.mark.parametrize("bits", [4, 8])
def test_a_request_from_projections_to_decoded_tokens(ctx, bits):
    """As a server runs them: norm and rotation of a prompt, the filtered prompt into a quantised cache, then for each token
    norm and rotation at the position the state has counted to, and the filtered step."""
    Bn, Hq, Hkv, n, steps, eta, tau0 = 2, 8, 2, 120, 24, 0.05, 0.4
    _say("cache request %d" % bits)
    w = synth.scaled(synth.workload(0), batch=Bn, seq=n + steps, n_q_heads=Hq, n_kv_heads=Hkv, dtype="bf16")
    q, k, v, _ = (x.cuda() if isinstance(x, torch.Tensor) else x for x in synth.make_qkv(w))
    freq = torch.exp(torch.arange(64, dtype=torch.float64, device="cuda") * (-np.log(1e4) / 64))
    wq, wk = (1 + 0.1 * torch.randn(128, device="cuda") for _ in range(2))
    whole = B.make_params(tuple(q.shape), tuple(k.shape), q.dtype, 0.5, 4)
    qr, kr = torch.empty_like(q), torch.empty_like(k)          # all tokens at once
    ctx.tf_norm_rotate(whole, B.make_rotary(freq, 128, wq, wk), q, k, qr, kr)
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), q.dtype, 0.5, 4)
    buf = B.DecodeBuffers(p, n + steps, cache_format=bits)
    a = [x[:, :, :n].contiguous() for x in (q, k, v)]
    ctx.tf_norm_rotate(p, B.make_rotary(freq, 128, wq, wk), a[0], a[1], a[0], a[1])
    keep, count = torch.empty((Bn, n), dtype=torch.uint8, device="cuda"), torch.empty(Bn, dtype=torch.int32, device="cuda")
    idx, fused, O = torch.empty((Bn, n), dtype=torch.int32, device="cuda"), torch.empty((Bn, n), device="cuda"), torch.empty_like(a[0])
    ctx.tf_decode_prefill_q(p, eta, tau0, buf.state, bits, *a, keep, idx, count, fused, O,
                            torch.empty(B.tf_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(a[0], qr[:, :, :n]) and torch.equal(a[1], kr[:, :, :n])
    kept = [keep[b].nonzero().flatten().tolist() for b in range(Bn)]
    one = B.make_params((Bn, Hq, 1, 128), (Bn, Hkv, 1, 128), q.dtype, 0.5, 4)
    rot = B.make_rotary(freq, 128, wq, wk, start=buf.seen)
    attended = 0
    for t in range(n, n + steps):
        a = [x[:, :, t].contiguous() for x in (q, k, v)]
        ctx.tf_norm_rotate(one, rot, a[0], a[1], a[0], a[1])
        ctx.tf_decode_step_q(p, eta, buf.state, bits, *a, buf.o, buf.skip, buf.fused, buf.ws)
        torch.cuda.synchronize()
        assert torch.equal(a[0], qr[:, :, t]) and torch.equal(a[1], kr[:, :, t])
        for b in range(Bn):
            if buf.skip[b]:
                assert not buf.o[b].any()
                continue
            kept[b].append(t)
            attended += 1
            kk, vv = (torch.from_numpy(ref.values(*ref.quantise(_f64(x[b][:, kept[b]]), bits), bits)).cuda()[None] for x in (kr, v))
            _check_attention(buf.o[b:b + 1, :, None], ref.attend(a[0][b:b + 1, :, None].double(), kk, vv, [len(kept[b])], [1], 128 ** -0.5), "bf16")
    assert 0 < attended < steps * Bn and buf.cache_len.tolist() == [len(x) for x in kept]


@pytest.mark.parametrize("case", [   # dtype, bits, batch, query heads, KV heads, prompt, steps, fusion, gamma
    ("bf16", 4, 2, 8, 2, 150, 40, B.TF_FUSE_EQ2, None), ("bf16", 8, 1, 32, 32, 65, 30, B.TF_FUSE_EQ2, 0.9),
    ("f32", 4, 3, 4, 4, 90, 25, B.TF_FUSE_KEY_ONLY, None), ("f32", 8, 2, 6, 2, 64, 20, B.TF_FUSE_INVVAR, None),
    ("bf16", 4, 1, 40, 40, 0, 70, B.TF_FUSE_EQ2, None), ("bf16", 4, 2, 128, 128, 30, 10, B.TF_FUSE_EQ2, None)])
def test_decoding_on_a_quantised_cache(ctx, case):
    """Scores, decisions, anchors and counters are those of the same calls on whole rows bit for bit; the caches hold the
    kept rows quantised; a token attends over what they stand for."""
    dt, bits, Bn, Hq, Hkv, n, steps, fusion, gamma = case
    _say("decode on a quantised cache %s" % (case,))
    eta, tau0, total = 0.05, 0.5, n + steps
    w = synth.scaled(synth.workload(0), batch=Bn, seq=total, n_q_heads=Hq, n_kv_heads=Hkv, dtype=dt)
    q, k, v, _ = (x.cuda() if isinstance(x, torch.Tensor) else x for x in synth.make_qkv(w))
    shape = (Bn, Hq, max(n, 1), 128), (Bn, Hkv, max(n, 1), 128)
    p = B.make_params(*shape, DT[dt], 0.5, 4, fusion, ema_gamma=gamma)
    plain, quant = B.DecodeBuffers(p, total), B.DecodeBuffers(p, total, cache_format=bits)
    quant.k_cache.fill_(0xFF)
    quant.v_cache.fill_(0xFF)
    kept = [[] for _ in range(Bn)]
    if n:
        outs = []
        for buf in (plain, quant):
            o = dict(keep=torch.empty((Bn, n), dtype=torch.uint8, device="cuda"),
                     kept_idx=torch.empty((Bn, n), dtype=torch.int32, device="cuda"),
                     count=torch.empty(Bn, dtype=torch.int32, device="cuda"),
                     fused=torch.empty((Bn, n), device="cuda"), O=torch.empty((Bn, Hq, n, 128), dtype=DT[dt], device="cuda"))
            args = [x[:, :, :n].contiguous() for x in (q, k, v)]
            ws = torch.empty(B.tf_workspace_bytes(p), dtype=torch.uint8, device="cuda")
            if buf is plain:
                ctx.tf_decode_prefill(p, eta, tau0, buf.state, *args, *o.values(), ws)
            else:
                ctx.tf_decode_prefill_q(p, eta, tau0, buf.state, bits, *args, *o.values(), ws)
            torch.cuda.synchronize()
            outs.append(o)
        for name in outs[0]:
            assert torch.equal(outs[0][name], outs[1][name]), name
        for b in range(Bn):
            kept[b] = outs[0]["keep"][b].nonzero().flatten().tolist()
    else:
        for buf in (plain, quant):
            ctx.tf_decode_init(p, buf.state, tau0)
    skipped = 0
    for t in range(n, total):
        a = [x[:, :, t].contiguous() for x in (q, k, v)]
        quant.ws.fill_(0xFF)
        quant.o.fill_(float("nan"))
        ctx.tf_decode_step(p, eta, plain.state, *a, plain.o, plain.skip, plain.fused, plain.ws)
        ctx.tf_decode_step_q(p, eta, quant.state, bits, *a, quant.o, quant.skip, quant.fused, quant.ws)
        torch.cuda.synchronize()
        for name in ("skip", "fused", "tau", "seen", "skipped", "cache_len", "overflow", "anchor_k", "anchor_v"):
            assert torch.equal(getattr(plain, name), getattr(quant, name)), (t, name)
        for b in range(Bn):
            if quant.skip[b]:
                skipped += 1
                assert not quant.o[b].any()
            else:
                kept[b].append(t)
        if t % 7 == 0 or t == total - 1:
            for b in range(Bn):
                if quant.skip[b]:
                    continue
                kk, vv = (torch.from_numpy(ref.values(*ref.quantise(_f64(x[b][:, kept[b]]), bits), bits)).cuda()[None] for x in (k, v))
                m = len(kept[b])
                _check_attention(quant.o[b:b + 1, :, None], ref.attend(a[0][b:b + 1, :, None].double(), kk, vv, [m], [1], 128 ** -0.5), dt)
    assert 0 < skipped < steps * Bn
    for t, x, is_value in ((quant.k_cache, k, False), (quant.v_cache, v, True)):
        code, ex = ref.unpack(_blob(t, Bn, Hkv, bits), bits, is_value)
        for b in range(Bn):
            m = len(kept[b])
            want = ref.quantise(_f64(x[b][:, kept[b]]), bits)
            np.testing.assert_array_equal(code[b, :, :m], want[0])
            np.testing.assert_array_equal(ex[b, :, :m], want[1])
            assert (code[b, :, m:] == (15 if bits == 4 else 255)).all() and (ex[b, :, m:] == 255).all()


def test_full_quantised_cache_sets_overflow(ctx):
    _say("decode quantised overflow")
    p = B.make_params((1, 2, 1, 128), (1, 2, 1, 128), torch.bfloat16, 0.5, 0)
    buf = B.DecodeBuffers(p, 3, cache_format=4)
    buf.k_cache.fill_(0xEE)
    ctx.tf_decode_init(p, buf.state, 50.0)       # nothing is skipped by the rule
    a = [_rows((1, 2, 128), "bf16", s) for s in range(3)]
    for t in range(5):
        ctx.tf_decode_step_q(p, 0.0, buf.state, 4, *a, buf.o, buf.skip, buf.fused, buf.ws)
        torch.cuda.synchronize()
        assert buf.skip.item() == (t >= 3) and buf.overflow.item() == (t >= 3) and buf.cache_len.item() == min(t + 1, 3)
        assert buf.o.any().item() == (t < 3)
    code, _ = ref.unpack(_blob(buf.k_cache, 1, 2, 4), 4, False)
    assert (code[:, :, 3:] == 0xE).all()


def test_refusals(ctx):
    _say("cache refusals")
    p = _params("bf16", 2, 4, 2, 8)
    c = B.QuantCache(p, 64, 4)
    k, v = (_rows((2, 2, 8, 128), "bf16", s) for s in (1, 2))
    q, o = _rows((2, 4, 8, 128), "bf16", 3), torch.zeros((2, 4, 8, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")

    def refused(f, *args, status=B.TF_ERR_INVALID_ARG):
        with pytest.raises(B.TokfiltError) as e:
            f(*args)
        assert e.value.status == status and len(str(e.value)) > 20

    for field, bad in (("format", 0), ("format", 5), ("capacity", 0), ("k", None), ("v", None), ("len", None),
                       ("k", c.k.data_ptr() + 8)):
        d = B.tf_cache(c.desc.k, c.desc.v, c.desc.len, c.desc.overflow, c.desc.capacity, c.desc.format)
        setattr(d, field, bad)
        refused(ctx.tf_cache_write, p, d, k, v, None, 8, None)
        refused(ctx.tf_cache_read, p, d, None, k, v)
        refused(ctx.tf_cache_attend, p, d, q, o, None, ws)
    for m in (0, -1, 9):
        refused(ctx.tf_cache_write, p, c.desc, k, v, None, m, None)
    refused(ctx.tf_cache_write, p, c.desc, None, v, None, 8, None)
    refused(ctx.tf_cache_write, p, c.desc, k.view(-1)[4:], v, None, 8, None)
    refused(ctx.tf_cache_read, p, c.desc, None, k, None)
    refused(ctx.tf_cache_attend, p, c.desc, q, None, None, ws)
    refused(ctx.tf_cache_attend, p, c.desc, q, q, None, ws)
    refused(ctx.tf_cache_attend, p, c.desc, q, o, None, None)
    folded = _params("bf16", 2, 4, 2, 8, kv_stride=(0, 1024, 128), o_stride=(4096, 0, 128))
    refused(ctx.tf_cache_read, folded, c.desc, None, k, v)
    refused(ctx.tf_cache_attend, folded, c.desc, q, o, None, ws)
    big = B.make_params((1, 8, 8, 128), (1, 2, 8, 128), torch.bfloat16, 0.0)
    need = B.tf_cache_workspace_bytes(big)
    cb = B.QuantCache(big, 5000, 4)
    refused(ctx.tf_cache_attend, big, cb.desc, _rows((1, 8, 8, 128), "bf16", 1), torch.empty((1, 8, 8, 128), dtype=torch.bfloat16, device="cuda"),
            None, torch.empty(16, dtype=torch.uint8, device="cuda"), status=B.TF_ERR_WORKSPACE_TOO_SMALL)
    assert need > 16
    buf = B.DecodeBuffers(p, 8, cache_format=4)
    a = [_rows((2, h, 128), "bf16", 4) for h in (4, 2, 2)]
    refused(ctx.tf_decode_step_q, p, 0.0, buf.state, 3, *a, buf.o, buf.skip, buf.fused, buf.ws)
    refused(ctx.tf_decode_step_q, p, -1.0, buf.state, 4, *a, buf.o, buf.skip, buf.fused, buf.ws)
    refused(ctx.tf_decode_prefill_q, p, 0.0, 0.5, buf.state, 7, q, k, v, None, None, None, None, o, ws)
    torch.cuda.synchronize()
    assert not o.any() and c.len.tolist() == [0, 0]
