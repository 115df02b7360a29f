"""Columns that are not rotated, without norms, are passed on bit for bit, whatever they hold, and reach no other column."""
import pytest
import torch

from paper_2512_07090_amd import binding as B
from test_gpu_norm_rotate import DT, EPS, _check, _freq, _reference, _rows, ctx  # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot_dim", [0, 16, 96])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", [("bf16", 2, 5, 5, 3), ("f32", 1, 17, 17, 700)])
def test_passed_on(ctx, case, interleaved, rot_dim):  # noqa: F811
    dt, Bn, Hq, Hkv, n = case
    print("[case] passed on %s %s %d" % (case, interleaved, rot_dim), flush=True)
    q, k = (_rows((Bn, h, n, 128), dt, s) for h, s in ((Hq, 1), (Hkv, 2)))
    for x in (q, k):
        special = torch.tensor([float("inf"), -0.0, float("-inf"), 1.0, float("nan"), -0.0, 0.0, -1.0], device="cuda").to(x.dtype)
        x[..., 100:108] = special
    pos = torch.arange(n, device="cuda").expand(Bn, n)
    freq = _freq(rot_dim) if rot_dim else None
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), DT[dt], 0.0)
    out = [torch.zeros_like(x) for x in (q, k)]
    ctx.tf_norm_rotate(p, B.make_rotary(freq, rot_dim, eps=EPS, interleaved=interleaved), q, k, *out)
    torch.cuda.synchronize()
    bits = torch.int32 if dt == "f32" else torch.int16
    for o, x in zip(out, (q, k)):
        assert torch.equal(o[..., rot_dim:].contiguous().view(bits), x[..., rot_dim:].contiguous().view(bits))
        r, mag = _reference(x, None, pos, freq, rot_dim, interleaved)
        _check(o[..., :rot_dim], (r[..., :rot_dim], mag[..., :rot_dim]), dt)
