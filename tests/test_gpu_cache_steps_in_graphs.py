"""Decoded tokens over quantised caches from replayed graphs: norm and rotation at the position that the state has counted to,
then the filtered step, two layers over one workspace, against the same calls made one by one.  Equal bit for bit."""
import pytest
import torch

from paper_2512_07090_amd import binding as B
from test_gpu_cache import DT, _rows, ctx  # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [("bf16", 4, 2, 8, 2, 1500), ("f32", 8, 3, 4, 4, 700), ("bf16", 8, 1, 40, 40, 130)])
def test_steps_from_replayed_graphs(ctx, case):  # noqa: F811
    dt, bits, Bn, Hq, Hkv, n = case
    print("[case] steps in graphs %s" % (case,), flush=True)
    steps, layers = 8, 2
    p = B.make_params((Bn, Hq, n, 128), (Bn, Hkv, n, 128), DT[dt], 0.5, 4)
    one = B.make_params((Bn, Hq, 1, 128), (Bn, Hkv, 1, 128), DT[dt], 0.5, 4)
    freq = torch.exp(torch.arange(64, dtype=torch.float64, device="cuda") * -0.14)

    def prompt(layer):
        buf = B.DecodeBuffers(p, n + steps, cache_format=bits)
        q, k, v = (_rows((Bn, h, n, 128), dt, 10 * layer + s, 0.2) for s, h in enumerate((Hq, Hkv, Hkv)))
        keep, count = torch.empty((Bn, n), dtype=torch.uint8, device="cuda"), torch.empty(Bn, dtype=torch.int32, device="cuda")
        idx, fused = torch.empty((Bn, n), dtype=torch.int32, device="cuda"), torch.empty((Bn, n), device="cuda")
        ctx.tf_decode_prefill_q(p, 0.05, 0.0, buf.state, bits, q, k, v, keep, idx, count, fused, torch.empty_like(q),
                                torch.empty(B.tf_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
        return buf

    tokens = [[[_rows((Bn, h, 128), dt, 1000 + 100 * layer + 3 * t + s, 0.2) for s, h in enumerate((Hq, Hkv, Hkv))] for t in range(steps)]
              for layer in range(layers)]

    def call(buf, rot, q, k, v, ws):
        ctx.tf_norm_rotate(one, rot, q, k, q, k)
        ctx.tf_decode_step_q(one, 0.05, buf.state, bits, q, k, v, buf.o, buf.skip, buf.fused, ws)

    want = [[] for _ in range(layers)]
    for layer in range(layers):
        buf = prompt(layer)
        rot = B.make_rotary(freq, 128, start=buf.seen)
        for t in range(steps):
            q, k, v = (x.clone() for x in tokens[layer][t])
            call(buf, rot, q, k, v, buf.ws)
            torch.cuda.synchronize()
            want[layer].append([x.clone() for x in (buf.o, buf.skip, buf.fused, buf.tau, buf.cache_len, buf.seen)])

    ws = torch.full((B.tf_cache_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    bufs = [prompt(layer) for layer in range(layers)]
    rots = [B.make_rotary(freq, 128, start=buf.seen) for buf in bufs]
    held = [[torch.empty_like(x) for x in tokens[layer][0]] for layer in range(layers)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(layers)]
    for layer, g in enumerate(graphs):
        with torch.cuda.graph(g, stream=s):
            call(bufs[layer], rots[layer], *held[layer], ws)
    skipped = 0
    for t in range(steps):
        for layer in range(layers):
            for x, y in zip(held[layer], tokens[layer][t]):
                x.copy_(y)
            if t % 3 == 2:
                ws.fill_(t)                    # between calls the workspace is whoever's
            graphs[layer].replay()
            torch.cuda.synchronize()
            buf = bufs[layer]
            skipped += int(buf.skip.sum())
            for got, w in zip((buf.o, buf.skip, buf.fused, buf.tau, buf.cache_len, buf.seen), want[layer][t]):
                assert torch.equal(got, w), (t, layer)
    assert skipped < steps * layers * Bn
