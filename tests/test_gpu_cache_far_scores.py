"""Scores as far from zero as fp32 holds them: a softmax only knows differences.

A key is its own power of two in column 0 and a query a number there, so that a score before its scaling is exact.  Keys that
are equal have equal scores and equal weights, so that the output is the mean of their values: of at most 4 values of +-1 and
+-2, sums and quotients of which are exact in bf16, and within 2^-22 in fp32 (a sum of equal weights, a quotient).  Other keys
are smaller or larger by 2^20, and their scores differ by more than any exponent holds: all weight is on the largest."""
import pytest
import torch

from paper_2512_07090_amd import binding as B
from test_gpu_cache import DT, _params, ctx  # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [   # dtype, batch, heads, KV heads, keys, new tokens: one query a form; slices; many columns
    ("bf16", 2, 2, 1, 1, 1), ("f32", 2, 2, 1, 4, 1), ("bf16", 1, 12, 1, 4, 1), ("bf16", 1, 4, 2, 700, 1), ("f32", 1, 1, 1, 1300, 1),
    ("bf16", 16, 8, 8, 70, 70)])
@pytest.mark.parametrize("far", [(-1.0, 35), (-1.0, 125), (-1.6875, 44), (1.6875, 35), (-1.171875, 105), (1.171875, 123)])
def test_far_scores(ctx, case, bits, far):  # noqa: F811
    dt, Bn, Hq, Hkv, m, n = case
    number, e = far
    print("[case] far scores %s %d %s" % (case, bits, far), flush=True)
    p, pm = _params(dt, Bn, Hq, Hkv, n, softmax_scale=0.11), _params(dt, Bn, Hkv, Hkv, m)
    k, v = (torch.zeros((Bn, Hkv, m, 128), dtype=DT[dt], device="cuda") for _ in range(2))
    few = min(m, 4)                                     # the first rows have the largest scores
    k[..., 0] = 2.0 ** (e if number < 0 else e - 20)
    k[:, :, :few, 0] = 2.0 ** (e - 20 if number < 0 else e)
    sign = torch.tensor([1.0, 2.0, -2.0, 1.0], device="cuda")[:few].to(DT[dt])
    v[:, :, :few] = sign[:, None]
    v[:, :, few:] = 3.0
    q = torch.zeros((Bn, Hq, n, 128), dtype=DT[dt], device="cuda")
    q[..., 0] = number
    c = B.QuantCache(p, m, bits)
    ctx.tf_cache_write(pm, c.desc, k, v, None, m, None)
    o = torch.full_like(q, float("nan"))
    ctx.tf_cache_attend(p, c.desc, q, o, None, torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for t in range(n):
        seen = min(few, m - n + t + 1)
        mean = (sign[:seen].double().sum() / seen).to(DT[dt]).double()
        assert ((o[:, :, t].double() - mean).abs() <= (2.0 ** -22 * mean.abs() if dt == "f32" else 0)).all(), t


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("case", [("bf16", 1, 2, 1), ("f32", 2, 2, 2), ("bf16", 1, 12, 1)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_small_differences_of_large_scores(ctx, case, bits, sign):  # noqa: F811
    """Scores of 2^23 and i more, exact in fp32, times 4 log2(e): their differences are what the weights know.  An exponent is
    then off by one rounding of a number below 18 (2^-20), a bf16 weight by its two parts (2^-16), sums by less than 2^-18:
    fp32 |o - ref| <= 2^-17 A, bf16 2^-14 A + 2^-8 |ref|, A the weighted sum of |v|."""
    dt, Bn, Hq, Hkv = case
    print("[case] small differences %s %d %g" % (case, bits, sign), flush=True)
    m = 4
    p, pm = _params(dt, Bn, Hq, Hkv, 1, softmax_scale=4.0), _params(dt, Bn, Hkv, Hkv, m)
    k, v = (torch.zeros((Bn, Hkv, m, 128), dtype=DT[dt], device="cuda") for _ in range(2))
    i = torch.arange(m, device="cuda").to(DT[dt])
    k[..., 0], k[..., 32] = 2.0 ** 23, i
    v[..., :32], v[..., 32:] = (2 - i)[:, None], torch.tensor([1.0, 4.0, 2.0, -1.0], device="cuda").to(DT[dt])[:, None]
    q = torch.zeros((Bn, Hq, 1, 128), dtype=DT[dt], device="cuda")
    q[..., 0], q[..., 32] = sign, 1.0
    c = B.QuantCache(p, m, bits)
    ctx.tf_cache_write(pm, c.desc, k, v, None, m, None)
    o = torch.full_like(q, float("nan"))
    ctx.tf_cache_attend(p, c.desc, q, o, None, torch.empty(B.tf_cache_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    w = torch.softmax(4 * i.double(), 0)
    ref, A = w @ v[0, 0].double(), w @ v[0, 0].double().abs()
    tol = 2.0 ** -17 * A if dt == "f32" else 2.0 ** -14 * A + 2.0 ** -8 * ref.abs()
    assert ((o[:, :, 0].double() - ref).abs() <= tol).all()
