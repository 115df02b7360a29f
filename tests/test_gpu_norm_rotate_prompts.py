"""Norm and rotation of prompts: calls long enough for workgroups of four tokens, and for results that go past the caches.
Same formula in 64 bits and same tolerance as for short calls."""
import pytest
import torch

from paper_2512_07090_amd import binding as B
from test_gpu_norm_rotate import DT, EPS, _check, _freq, _reference, _rows, ctx  # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def _say(msg):
    print("[case] " + msg, flush=True)


def _form(dt, Bn, Hq, Hkv, n):
    """What the launcher chooses: one token a workgroup, four, or four with results past the caches."""
    parts = -(-Hq // 16) + -(-Hkv // 16)
    if n < 4 or Bn * n * parts <= 2048:
        return "one"
    return "stream" if (8 if dt == "f32" else 4) * Bn * n * 128 * (Hq + Hkv) > 1 << 28 else "four"


def _run(ctx, dt, Bn, Hq, Hkv, n, rot_dim, interleaved, norm, positions, layout):
    x = []
    for h, seed, by_token in ((Hq, 1, layout in ("tokens", "mixed")), (Hkv, 2, layout == "tokens")):
        t = _rows((Bn, n, h, 128), dt, seed)
        x.append(t.transpose(1, 2) if by_token else t.transpose(1, 2).contiguous())
    g = torch.Generator(device="cuda").manual_seed(3)
    wq, wk = (1 + 0.3 * torch.randn(128, generator=g, device="cuda") for _ in range(2)) if norm else (None, None)
    given = torch.randint(-1000, 200000, (Bn, n), generator=g, device="cuda").int() if positions else None
    start = torch.tensor([5 + 1001 * b for b in range(Bn)], dtype=torch.int32, device="cuda")
    pos = (given.long() if positions else torch.arange(n, device="cuda").expand(Bn, n)) + start.long()[:, None]
    freq = _freq(rot_dim) if rot_dim else None
    rot = B.make_rotary(freq, rot_dim, wq, wk, given, start, EPS, interleaved)
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), DT[dt], 0.0, q_stride=x[0].stride()[:3],
                      kv_stride=x[1].stride()[:3], o_stride=x[0].stride()[:3])
    want = [_reference(t, w, pos, freq, rot_dim, interleaved) for t, w in zip(x, (wq, wk))]
    out = x if layout == "in place" else [torch.full_like(t, float("nan")) for t in x]
    ctx.tf_norm_rotate(p, rot, x[0], x[1], out[0], out[1])
    torch.cuda.synchronize()
    for o, w in zip(out, want):
        _check(o, w, dt)


@pytest.mark.parametrize("case", [   # dtype, batch, query heads, KV heads, n, rot_dim, interleaved, norm, positions, form
    ("bf16", 1, 32, 8, 682, 128, False, True, False, "one"), ("bf16", 1, 32, 8, 683, 128, False, True, False, "four"),
    ("bf16", 2, 40, 40, 203, 64, True, True, True, "four"), ("f32", 3, 17, 1, 463, 128, False, True, False, "four"),
    ("f32", 3, 17, 1, 461, 112, True, False, True, "four"), ("bf16", 5, 24, 8, 150, 32, False, True, True, "four"),
    ("bf16", 2, 8, 1, 514, 0, False, True, False, "four"), ("f32", 1, 5, 5, 1026, 96, False, True, False, "four"),
    ("bf16", 300, 16, 16, 4, 128, False, True, False, "four"), ("f32", 200, 33, 11, 5, 16, True, True, False, "four"),
    ("bf16", 700, 6, 3, 3, 128, False, True, False, "one")])
@pytest.mark.parametrize("layout", ["rows", "tokens", "mixed", "in place"])
def test_prompts_match_64_bits(ctx, case, layout):  # noqa: F811
    *shape, form = case
    _say("norm and rotation of a prompt %s %s" % (case, layout))
    assert _form(*shape[:5]) == form
    _run(ctx, *shape, layout)


@pytest.mark.parametrize("case", [("bf16", 1, 32, 32, 8193, 128, False, True, False), ("f32", 2, 40, 40, 1639, 64, True, True, True)])
@pytest.mark.parametrize("layout", ["rows", "tokens", "in place"])
def test_results_past_the_caches_match_64_bits(ctx, case, layout):  # noqa: F811
    _say("norm and rotation past the caches %s %s" % (case, layout))
    assert _form(*case[:5]) == "stream"
    _run(ctx, *case, layout)


def test_one_tensor_of_a_long_prompt(ctx):  # noqa: F811
    """Queries alone, then keys alone: a token's workgroups are those of one tensor."""
    Bn, Hq, Hkv, n = 2, 20, 5, 1027
    _say("norm and rotation, one tensor of a prompt")
    assert _form("bf16", Bn, 0, Hkv, n) == "four"
    q, k = _rows((Bn, Hq, n, 128), "bf16", 4), _rows((Bn, Hkv, n, 128), "bf16", 5)
    w = torch.rand(128, device="cuda") + 0.5
    pos = torch.arange(n, device="cuda").expand(Bn, n)
    rot = B.make_rotary(_freq(128), 128, w, w, eps=EPS)
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), torch.bfloat16, 0.0)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    ctx.tf_norm_rotate(p, rot, q, None, qo, None)
    ctx.tf_norm_rotate(p, rot, None, k, None, ko)
    torch.cuda.synchronize()
    _check(qo, _reference(q, w, pos, _freq(128), 128, False), "bf16")
    _check(ko, _reference(k, w, pos, _freq(128), 128, False), "bf16")
