"""What a NaN or an infinity becomes in a cache of 4 or 8 bits: its block of 32 columns reads back as NaN, and so does what
is computed from it; everything else of the cache is as without it.  No tolerances: bytes, and values that codes stand for.
"""
import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_2512_07090_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BAD = (float("nan"), float("inf"), float("-inf"))


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


def _rows(shape, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dt])


def _spoil(x, seed):
    """x [..., 128] with one element in about a third of its rows not finite; which blocks [..., 4] that are."""
    g = np.random.default_rng(seed)
    y = x.clone()
    flat = y.view(-1, 128)
    hit = np.zeros((flat.shape[0], 4), bool)
    for i in range(flat.shape[0]):
        if g.random() < 0.35 or i == 0:
            col = int(g.integers(128))
            flat[i, col] = BAD[int(g.integers(3))]
            hit[i, col // 32] = True
    return y, torch.from_numpy(hit.reshape(tuple(x.shape[:-1]) + (4,)))


def _check(code, ex, clean, hit, bits):
    """Codes and exponents of rows against those of the rows without what was spoilt."""
    want_c, want_e = ref.quantise(clean.double().cpu().numpy(), bits)
    hit = hit.numpy()
    assert (ex[hit] == 255).all()
    np.testing.assert_array_equal(ex[~hit], want_e[~hit])
    blocks = lambda c: c.reshape(c.shape[:-1] + (4, 32))
    np.testing.assert_array_equal(blocks(code)[~hit], blocks(want_c)[~hit])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [("bf16", 1, 2, 3), ("f32", 2, 2, 5), ("bf16", 2, 3, 200), ("f32", 1, 4, 130)])
def test_written_and_read_back(ctx, case, bits):
    """Few rows (one workgroup for all of a batch row) and many (one for each page)."""
    dt, Bn, Hkv, n = case
    _say("cache not finite %s %d" % (case, bits))
    p = _params(dt, Bn, Hkv, Hkv, n)
    c = B.QuantCache(p, n + 9, bits)
    clean = [_rows((Bn, Hkv, n, 128), dt, s) for s in (1, 2)]
    (k, hk), (v, hv) = _spoil(clean[0], 3), _spoil(clean[1], 4)
    ctx.tf_cache_write(p, c.desc, k, v, None, n, None)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    ctx.tf_cache_read(p, c.desc, None, ko, vo)
    torch.cuda.synchronize()
    for t, o, x, hit, is_value in ((c.k, ko, clean[0], hk, False), (c.v, vo, clean[1], hv, True)):
        blob = t.cpu().numpy().reshape(Bn, Hkv, -1, ref.page_bytes(bits))
        code, ex = ref.unpack(blob, bits, is_value)
        _check(code[:, :, :n], ex[:, :, :n], x, hit, bits)
        want = torch.from_numpy(ref.values(*ref.quantise(x.double().cpu().numpy(), bits), bits))
        got = o.double().cpu().view(Bn, Hkv, n, 4, 32)
        assert torch.isnan(got[hit]).all()
        assert torch.equal(got[~hit], want.view(Bn, Hkv, n, 4, 32)[~hit])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_prompt_and_a_step_leave_the_bytes_that_a_write_leaves(ctx, dt, bits):
    """Values that are not finite (the filter reads keys alone here, so its decisions are defined); nothing is skipped."""
    Bn, H, n = 2, 3, 70
    _say("prompt and steps, not finite %s %d" % (dt, bits))
    p = B.make_params((Bn, H, n, 128), (Bn, H, n, 128), DT[dt], 0.5, 0, B.TF_FUSE_KEY_ONLY)
    q, k, clean = (_rows((Bn, H, n + 6, 128), dt, s) for s in (5, 6, 7))
    v, hit = _spoil(clean, 8)
    buf = B.DecodeBuffers(p, n + 6, cache_format=bits)
    a = [x[:, :, :n].contiguous() for x in (q, k, v)]
    keep, count = torch.empty((Bn, n), dtype=torch.uint8, device="cuda"), torch.empty(Bn, dtype=torch.int32, device="cuda")
    idx, fused = torch.empty((Bn, n), dtype=torch.int32, device="cuda"), torch.empty((Bn, n), device="cuda")
    ctx.tf_decode_prefill_q(p, 0.0, 50.0, buf.state, bits, *a, keep, idx, count, fused, torch.empty_like(a[0]),
                            torch.empty(B.tf_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    for t in range(n, n + 6):
        a = [x[:, :, t].contiguous() for x in (q, k, v)]
        ctx.tf_decode_step_q(p, 0.0, buf.state, bits, *a, buf.o, buf.skip, buf.fused, buf.ws)
    one = _params(dt, Bn, H, H, n + 6)
    c = B.QuantCache(one, n + 6, bits)
    ctx.tf_cache_write(one, c.desc, k, v, None, n + 6, None)
    torch.cuda.synchronize()
    assert buf.cache_len.tolist() == [n + 6] * Bn
    for t, w, x, h, is_value in ((buf.v_cache, c.v, clean, hit, True), (buf.k_cache, c.k, k, torch.zeros_like(hit), False)):
        code, ex = (y[:, :, :n + 6] for y in ref.unpack(t.cpu().numpy().reshape(Bn, H, -1, ref.page_bytes(bits)), bits, is_value))
        _check(code, ex, x, h, bits)
        code2, ex2 = (y[:, :, :n + 6] for y in ref.unpack(w.cpu().numpy().reshape(Bn, H, -1, ref.page_bytes(bits)), bits, is_value))
        np.testing.assert_array_equal(code, code2)
        np.testing.assert_array_equal(ex, ex2)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [   # dtype, batch, query heads, KV heads, new tokens, keys: one form of the kernel each
    ("bf16", 2, 4, 2, 1, 90), ("bf16", 2, 4, 2, 12, 700), ("f32", 2, 4, 2, 3, 130), ("bf16", 16, 8, 8, 70, 130)])
def test_a_query_that_sees_one_is_nan_and_no_other_cache_is(ctx, case, bits):
    dt, Bn, Hq, Hkv, n, m = case
    _say("cache attend, not finite %s %d" % (case, bits))
    p, pm = _params(dt, Bn, Hq, Hkv, n), _params(dt, Bn, Hkv, Hkv, m)
    k, v, q = (_rows((Bn, h, r, 128), dt, s) for h, r, s in ((Hkv, m, 9), (Hkv, m, 10), (Hq, n, 11)))
    ws = torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    outs = []
    for spoilt in (None, "key", "value"):
        k2, v2 = k.clone(), v.clone()
        # batch row 1, KV head 0, a row that every query of the call sees; columns 32 .. 63
        for i, bad in enumerate(BAD):
            if spoilt:
                (k2 if spoilt == "key" else v2)[1, 0, 5 * i, 40 + i] = bad
        c = B.QuantCache(p, m, bits)
        ctx.tf_cache_write(pm, c.desc, k2, v2, None, m, None)
        o = torch.zeros_like(q)
        ctx.tf_cache_attend(p, c.desc, q, o, None, ws)
        torch.cuda.synchronize()
        outs.append(o.float())
    hit = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
    hit[1, :Hq // Hkv] = True
    assert torch.isfinite(outs[0]).all()
    assert torch.isnan(outs[1][hit]).all() and torch.equal(outs[1][~hit], outs[0][~hit])
    hit[..., :32] = hit[..., 64:] = False
    assert torch.isnan(outs[2][hit]).all() and torch.equal(outs[2][~hit], outs[0][~hit])
