"""Norms of queries and keys and the position rotation through the C ABI, against the formula in 64 bits.

Tolerance: with (a, b) the normalised pair in 64 bits, a row's norm is off by at most some ten fp32 roundings (a sum of 128
squares in 12 additions, a root, a division, two products: 2^-20 of the value), cos and sin by 2^-22 (their argument is a
turn's part rounded to fp32, and a rounding of their own), the two products and their sum by 2^-23 more:
  fp32  |y - ref| <= 2^-19 (|a| + |b|)          bf16  + 2^-8 |ref|
"""
import math

import pytest
import torch

from paper_2512_07090_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c = B.Context(0)
    yield c
    c.close()


def _say(msg):
    print("[case] " + msg, flush=True)


def _rows(shape, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp(torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x.view(-1, 128)[0] = 0                         # a row of zeros
    return x.to(DT[dt])


def _freq(rot_dim, base=10000.0):
    half = rot_dim // 2
    return torch.exp(torch.arange(half, dtype=torch.float64, device="cuda") * (-math.log(base) / max(half, 1)))


def _reference(x, w, pos, freq, rot_dim, interleaved):
    """(result, |a| + |b|) in float64; pos int64 [B, n]."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * w.double()
    if rot_dim == 0:
        return y, y.abs()
    angle = (pos.double()[..., None] * freq)[:, None]
    c, s = torch.cos(angle), torch.sin(angle)
    i = torch.arange(rot_dim // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot_dim // 2)
    out, mag = y.clone(), y.abs()
    a, b = y[..., first], y[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    mag[..., first] = mag[..., second] = a.abs() + b.abs()
    return out, mag


def _check(got, want, dt):
    r, mag = want
    tol = 2.0 ** -19 * mag + (2.0 ** -8 * r.abs() if dt == "bf16" else 0)
    err = (got.double() - r).abs()
    assert (err <= tol).all(), (err - tol).max().item()


@pytest.mark.parametrize("case", [   # dtype, batch, query heads, KV heads, n, rot_dim, interleaved, norm, positions, start
    ("bf16", 1, 32, 8, 1, 128, False, True, None, 100003), ("bf16", 2, 5, 5, 7, 64, True, True, None, 0),
    ("f32", 2, 6, 2, 33, 128, False, True, "given", None), ("f32", 1, 4, 1, 5, 16, False, False, None, 2 ** 31 - 40),
    ("bf16", 3, 1, 1, 130, 0, False, True, None, None), ("f32", 1, 3, 3, 9, 128, True, False, "given", 5),
    ("bf16", 2, 40, 40, 66, 32, False, True, None, None), ("f32", 1, 2, 2, 4, 128, False, True, "negative", None),
    ("bf16", 1, 8, 8, 4, 96, False, True, None, 3), ("f32", 2, 4, 4, 11, 112, True, True, "given", 1)])
@pytest.mark.parametrize("layout", ["rows", "tokens", "in place"])
def test_matches_64_bits(ctx, case, layout):
    dt, Bn, Hq, Hkv, n, rot_dim, interleaved, norm, positions, start = case
    _say("norm and rotation %s %s" % (case, layout))
    x = []
    for h, seed in ((Hq, 1), (Hkv, 2)):
        t = _rows((Bn, n, h, 128), dt, seed)
        x.append(t.transpose(1, 2) if layout == "tokens" else t.transpose(1, 2).contiguous())
    g = torch.Generator(device="cuda").manual_seed(3)
    wq, wk = (1 + 0.3 * torch.randn(128, generator=g, device="cuda") for _ in range(2)) if norm else (None, None)
    pos = torch.arange(n, device="cuda").expand(Bn, n)
    given = None
    if positions:
        given = torch.randint(0, 2000, (Bn, n), generator=g, device="cuda").int()
        if positions == "negative":
            given -= 1000
        pos = given.long()
    st = None
    if start is not None:
        st = torch.tensor([start - 17 * b if b <= start // 17 else start for b in range(Bn)], dtype=torch.int32, device="cuda")
        pos = pos + st.long()[:, None]
    freq = _freq(rot_dim) if rot_dim else None
    rot = B.make_rotary(freq, rot_dim, wq, wk, given, st, EPS, interleaved)
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), DT[dt], 0.0, q_stride=x[0].stride()[:3],
                      kv_stride=x[1].stride()[:3], o_stride=x[0].stride()[:3])
    want = [_reference(t, w, pos, freq, rot_dim, interleaved) for t, w in zip(x, (wq, wk))]
    out = x if layout == "in place" else [torch.full_like(t, float("nan")) for t in x]
    ctx.tf_norm_rotate(p, rot, x[0], x[1], out[0], out[1])
    torch.cuda.synchronize()
    for o, w in zip(out, want):
        _check(o, w, dt)


def test_one_tensor_alone_and_strided_output(ctx):
    Bn, Hq, Hkv, n = 2, 4, 2, 10
    _say("norm and rotation, one tensor")
    q, k = _rows((Bn, Hq, n, 128), "bf16", 4), _rows((Bn, Hkv, n, 128), "bf16", 5)
    w = torch.rand(128, device="cuda") + 0.5
    pos = torch.arange(n, device="cuda").expand(Bn, n)
    rot = B.make_rotary(_freq(128), 128, w, w, eps=EPS)
    o = torch.full((Bn, n, Hq, 160), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = o[..., :128].transpose(1, 2)
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), torch.bfloat16, 0.0, o_stride=view.stride()[:3])
    ctx.tf_norm_rotate(p, rot, q, None, view, None)
    ko = torch.full_like(k, float("nan"))
    ctx.tf_norm_rotate(p, rot, None, k, None, ko)
    torch.cuda.synchronize()
    _check(view, _reference(q, w, pos, _freq(128), 128, False), "bf16")
    _check(ko, _reference(k, w, pos, _freq(128), 128, False), "bf16")
    assert torch.isnan(o[..., 128:]).all()


def test_replayed_graph_follows_the_positions(ctx):
    """A decoded token's position is read on the device: the captured call turns by it at every replay."""
    _say("norm and rotation, graph")
    Bn, Hq, Hkv = 3, 8, 2
    q, k = _rows((Bn, Hq, 1, 128), "bf16", 6), _rows((Bn, Hkv, 1, 128), "bf16", 7)
    seen = torch.zeros(Bn, dtype=torch.int32, device="cuda")
    rot = B.make_rotary(_freq(128), 128, start=seen, eps=EPS)
    p = B.make_params((Bn, Hq, 1, 128), (Bn, Hkv, 1, 128), torch.bfloat16, 0.0)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ctx.tf_norm_rotate(p, rot, q, k, qo, ko)
    for at in ([0, 1, 2], [500, 7, 100000], [3, 3, 3]):
        seen.copy_(torch.tensor(at, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        pos = seen.long()[:, None]
        _check(qo, _reference(q, None, pos, _freq(128), 128, False), "bf16")
        _check(ko, _reference(k, None, pos, _freq(128), 128, False), "bf16")


def test_refusals(ctx):
    _say("norm and rotation refusals")
    q, k = torch.zeros((1, 2, 4, 128), device="cuda"), torch.zeros((1, 2, 4, 128), device="cuda")
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    p = B.make_params((1, 2, 4, 128), (1, 2, 4, 128), torch.float32, 0.0)
    good = dict(freq=_freq(128), rot_dim=128, eps=EPS)

    def refused(p, rot, *args):
        with pytest.raises(B.TokfiltError) as e:
            ctx.tf_norm_rotate(p, rot, *args)
        assert e.value.status == B.TF_ERR_INVALID_ARG and len(str(e.value)) > 20

    for bad in (dict(rot_dim=24), dict(rot_dim=-16), dict(rot_dim=144), dict(freq=None), dict(eps=0.0), dict(eps=float("nan")),
                dict(eps=float("inf"))):
        refused(p, B.make_rotary(**dict(good, **bad)), q, k, qo, ko)
    rot = B.make_rotary(**good)
    for field, v in (("interleaved", 2), ("reserved", 1)):
        r = B.make_rotary(**good)
        setattr(r, field, v)
        refused(p, r, q, k, qo, ko)
    for args in ((None, None, None, None), (q, k, None, ko), (None, k, qo, ko), (q, None, qo, ko), (q.view(-1)[1:], k, qo, ko)):
        refused(p, rot, *args)
    moved = B.make_params((1, 2, 4, 128), (1, 2, 4, 128), torch.float32, 0.0, o_stride=(1024, 128, 256))
    refused(moved, rot, q, k, q, ko)                         # in place, but elsewhere
    refused(B.make_params((1, 2, 4, 128), (1, 2, 4, 128), torch.float32, 0.0, o_stride=(1024, 0, 128)), rot, q, k, qo, ko)
    with pytest.raises(B.TokfiltError):
        B.make_rotary(_freq(128).float(), 128)
    torch.cuda.synchronize()
    assert (qo == 5.0).all() and (ko == 5.0).all()
