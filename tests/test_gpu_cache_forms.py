"""Forms of the calls on a quantised cache that only some sizes choose: attention with two tiles of 16 columns by eight waves
(as many workgroups as compute units), with one of more than eight columns by four, and rows read back past the caches.
Tolerances and references are those of test_gpu_cache."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_2512_07090_amd import binding as B
from test_gpu_cache import DT, _check_attention, _params, _quant_cache, _rows, ctx  # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def _say(msg):
    print("[case] " + msg, flush=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [   # batch, query heads, KV heads, new tokens, lengths, counts, capacity
    (1, 32, 8, 256, [1111], None, 1200), (1, 32, 8, 256, [1111], [201], 1111), (1, 32, 8, 256, [100], [256], 130),
    (4, 32, 32, 49, [49, 640, 333, 0], None, 700), (4, 32, 32, 64, [700, 63, 64, 65], [64, 1, 0, 33], 700),
    (2, 64, 8, 64, [513, 2000], [64, 63], 2100)])
def test_attend_with_as_many_double_tiles_as_compute_units(ctx, case, bits):  # noqa: F811
    Bn, Hq, Hkv, n, lens, counts, cap = case
    _say("cache attend, 256 double tiles %s %d" % (case, bits))
    cols = n * (Hq // Hkv)
    assert Bn * Hkv * -(-cols // 16) >= 512 and Bn * Hkv * -(-cols // 32) == 256
    p = _params("bf16", Bn, Hq, Hkv, n)
    c, k, v = _quant_cache(p, "bf16", bits, Bn, Hkv, lens, cap, 120)
    q = _rows((Bn, Hq, n, 128), "bf16", 121, 0.2)
    o = torch.full_like(q, float("nan"))
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    ctx.tf_cache_attend(p, c.desc, q, o, cnt, ws)
    torch.cuda.synchronize()
    _check_attention(o, ref.attend(q.double(), k, v, lens, counts or [n] * Bn, 128 ** -0.5), "bf16", True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [   # batch, query heads, KV heads, new tokens, lengths, counts, capacity, most slices
    (40, 96, 8, 1, [13 * b for b in range(40)], None, 520, 1), (5, 384, 32, 1, [1100, 513, 1, 64, 900], None, 1100, 3),
    (5, 32, 32, 11, [11, 1090, 700, 5, 1024], [11, 3, 0, 5, 10], 1100, 3)])
def test_attend_of_nine_to_sixteen_columns_by_four_waves(ctx, case, bits):  # noqa: F811
    Bn, Hq, Hkv, n, lens, counts, cap, split = case
    _say("cache attend, four waves %s %d" % (case, bits))
    tiles = Bn * Hkv
    assert 8 < n * (Hq // Hkv) <= 16 and (tiles > 256 or 4 * tiles * (256 // tiles) <= 768)
    assert split == (1 if tiles > 256 else 512 // tiles)
    p = _params("bf16", Bn, Hq, Hkv, n)
    c, k, v = _quant_cache(p, "bf16", bits, Bn, Hkv, lens, cap, 125)
    q = _rows((Bn, Hq, n, 128), "bf16", 126, 0.2)
    o = torch.full_like(q, float("nan"))
    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    ctx.tf_cache_attend(p, c.desc, q, o, cnt, ws)
    torch.cuda.synchronize()
    _check_attention(o, ref.attend(q.double(), k, v, lens, counts or [n] * Bn, 128 ** -0.5), "bf16")


def test_many_caches_of_one_token_keep_weights_in_two_parts(ctx):  # noqa: F811
    """At most 16 columns a cache, whatever the number of caches: the tolerance is that of few queries."""
    Bn, Hq, Hkv = 64, 32, 8
    _say("cache attend, many caches of one token")
    lens = [30 + 9 * b for b in range(Bn)]
    p = _params("bf16", Bn, Hq, Hkv, 1)
    assert Bn * Hkv >= 512
    c, k, v = _quant_cache(p, "bf16", 4, Bn, Hkv, lens, 600, 130)
    q = _rows((Bn, Hq, 1, 128), "bf16", 131, 0.2)
    o = torch.full_like(q, float("nan"))
    ctx.tf_cache_attend(p, c.desc, q, o, None, torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    _check_attention(o, ref.attend(q.double(), k, v, lens, [1] * Bn, 128 ** -0.5), "bf16")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [("bf16", 2, 16, 16401), ("f32", 2, 16, 8203)])
def test_read_past_the_caches(ctx, case, bits):  # noqa: F811
    """Rows of a call above 256 MB, out of 997 different ones; from the middle of a cache, and behind its last row."""
    dt, Bn, Hkv, n = case
    _say("cache read past the caches %s %d" % (case, bits))
    assert 2 * (4 if dt == "f32" else 2) * 128 * Bn * Hkv * n > 1 << 28
    different = _rows((997, 128), dt, 140)
    value = torch.from_numpy(ref.values(*ref.quantise(different.double().cpu().numpy(), bits), bits)).cuda().to(DT[dt])
    b, h, i = (torch.arange(m, device="cuda").view(shape) for m, shape in ((Bn, (-1, 1, 1)), (Hkv, (1, -1, 1)), (n, (1, 1, -1))))
    which = [(29 * b + 13 * h + 7 * i + s) % 997 for s in (0, 500)]
    p = _params(dt, Bn, Hkv, Hkv, n)
    c = B.QuantCache(p, n, bits)
    held = [n, n - 70]
    ctx.tf_cache_write(p, c.desc, different[which[0]], different[which[1]], None, n, torch.tensor(held, dtype=torch.int32, device="cuda"))
    for start in ([0, 0], [1003, 64]):
        out = [torch.full((Bn, Hkv, n, 128), 77.0, dtype=DT[dt], device="cuda") for _ in range(2)]
        ctx.tf_cache_read(p, c.desc, torch.tensor(start, dtype=torch.int32, device="cuda"), *out)
        torch.cuda.synchronize()
        for o, w in zip(out, which):
            for row in range(Bn):
                there = held[row] - start[row]
                assert torch.equal(o[row, :, :there], value[w[row, :, start[row]:held[row]]])
                assert (o[row, :, there:] == 77.0).all()


def test_codes_below_bf16_are_cut_off(ctx):  # noqa: F811
    """fp32 rows near the smallest scale in 8 bits, read back as bf16: the upper halves of what the codes stand for."""
    print("[case] cache read, smallest codes", flush=True)
    n, H = 40, 2
    x = _rows((1, H, n, 128), "f32", 150) * 2.0 ** -130
    pf, pb = _params("f32", 1, H, H, n), _params("bf16", 1, H, H, n)
    c = B.QuantCache(pf, n, 8)
    ctx.tf_cache_write(pf, c.desc, x, x, None, n, None)
    f, b = (torch.zeros((1, H, n, 128), dtype=DT[dt], device="cuda") for dt in ("f32", "bf16"))
    ctx.tf_cache_read(pf, c.desc, None, f, f.clone())
    ctx.tf_cache_read(pb, c.desc, None, b, b.clone())
    torch.cuda.synchronize()
    want = torch.from_numpy(ref.values(*ref.quantise(x.double().cpu().numpy(), 8), 8))
    assert torch.equal(f.cpu().double(), want)
    assert torch.equal(b.view(torch.int16).int() & 0xFFFF, (f.view(torch.int32) >> 16) & 0xFFFF)
    assert not torch.equal(b.float(), f)
