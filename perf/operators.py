"""Performance cases of the operators around the filtered path, at the sizes a serving program calls them.

A case is one pass through public entry points of `paper_2512_07090_amd.binding`:

  kind "norm"    tf_norm_rotate: norms of queries and keys for each head and the position rotation
  kind "store"   tf_cache_write, then tf_cache_read: rows quantised behind what a cache holds, and read back
  kind "attend"  tf_cache_attend: new tokens attend over a cache held in 4 or 8 bits

Each has a plain form in elementary torch operations on the same inputs, and `exact` in 64 bits. A cache is the byte array
that include/tokfilt.h describes (pages of 64 rows: codes, then a scale for each row and 32 columns); the plain forms pack
and unpack it themselves.
"""
import math

import torch

own = False                # True: run() makes the framework's calls, else the plain form

DEVICE = "cuda:0"
D = 128                    # head size
BLOCK = 32                 # columns that share a scale
PAGE = 64                  # rows of a page
MHA_7B, MHA_13B, GQA_8B = (32, 32), (40, 40), (32, 8)   # (query heads, KV heads)
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


def _case(kind, dtype, batch, heads, n, **more):
    c = {"kind": kind, "dtype": dtype, "batch": batch, "n_q_heads": heads[0], "n_kv_heads": heads[1], "n": n, "bits": 4,
         "held": 0, "ratio": 0.0, "ragged": False, "rot_dim": 128, "interleaved": False, "norm": True, "first": 0,
         "by_token": False}
    c.update(more)
    return c


def listed():
    return [
        # a token that is being decoded, far into its context (smallest call)
        dict(_case("norm", "bf16", 1, GQA_8B, 1, first=100003), name="norm_gqa_b1_n1"),
        # the fp32 configuration, half of the columns rotated in neighbouring pairs
        dict(_case("norm", "f32", 1, MHA_7B, 512, rot_dim=64, interleaved=True), name="norm_f32_mha32_b1_n512"),
        # a full batch of prompts as the projections leave them, token by token
        dict(_case("norm", "bf16", 8, MHA_7B, 4096, by_token=True), name="norm_mha32_b8_n4096"),
        # one new token for each row of a batch
        dict(_case("store", "bf16", 8, GQA_8B, 1, held=2048), name="store_gqa_b8_n1"),
        # prompts of no round length under the feedback threshold: kept counts differ from row to row; 8 bits
        dict(_case("store", "bf16", 2, MHA_13B, 1777, bits=8, ratio=0.25, ragged=True), name="store_mha40_b2_n1777_fp8"),
        # a full batch of prompts, half of the tokens kept
        dict(_case("store", "bf16", 8, MHA_7B, 4096, ratio=0.5), name="store_mha32_b8_n4096"),
        # a token behind a short chat
        dict(_case("attend", "bf16", 1, GQA_8B, 1, held=500), name="attend_gqa_b1_c500"),
        # fp32 queries
        dict(_case("attend", "f32", 1, MHA_7B, 1, held=512, bits=8), name="attend_f32_mha32_b1_c512_fp8"),
        # steady decoding of a batch of medium-long sequences; 8 bits
        dict(_case("attend", "bf16", 8, MHA_7B, 1, held=2048, bits=8), name="attend_mha32_b8_c2048_fp8"),
        # one very long document
        dict(_case("attend", "bf16", 1, GQA_8B, 1, held=32768), name="attend_gqa_b1_c32768"),
        # a serving batch of long sequences of different length
        dict(_case("attend", "bf16", 16, GQA_8B, 1, held=16384, ragged=True), name="attend_gqa_b16_c16384"),
        # the next part of two prompts, in chunks (the last row's is shorter), over what is cached of them
        dict(_case("attend", "bf16", 2, GQA_8B, 256, held=6000, ragged=True), name="attend_gqa_b2_c6000_n256"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(("norm", "store", "attend", "attend"))
    heads = rng.choice((MHA_7B, MHA_13B, GQA_8B, (24, 8), (8, 1)))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    limit = max(_cost(c) for c in listed())
    while True:
        batch = rng.choice((1, 1, 2, 3, 5, 8, 16))
        if kind == "norm":
            c = _case(kind, dtype, batch, heads, _log_int(rng, 1, 16384), rot_dim=rng.choice((128, 128, 64, 32)),
                      interleaved=rng.random() < 0.3, norm=rng.random() < 0.75, by_token=rng.random() < 0.4,
                      first=rng.choice((0, _log_int(rng, 1, 1000000))))
            fits = batch * c["n"] <= 32768
        elif kind == "store":
            n = 1 if rng.random() < 0.25 else _log_int(rng, 2, 16384)
            c = _case(kind, dtype, batch, heads, n, bits=rng.choice((4, 8)), held=rng.choice((0, _log_int(rng, 1, 9000))),
                      ratio=0.0 if n == 1 else round(rng.uniform(0.0, 0.75), 3), ragged=n > 1 and rng.random() < 0.5)
            fits = batch * n <= 32768
        else:
            n = 1 if rng.random() < 0.6 else _log_int(rng, 2, 300)
            c = _case(kind, dtype, batch, heads, n, bits=rng.choice((4, 4, 8)), held=_log_int(rng, 30, 32768),
                      ragged=rng.random() < 0.5)
            c["held"] = max(c["held"], 2 * n)
            fits = batch * heads[1] * c["held"] <= 2 ** 21 and batch * heads[0] * n * c["held"] <= 2 ** 26
        if fits and _cost(c) <= limit:
            return c


# ------------------------------------------------------------------------------ inputs

def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _counts(case):
    """Rows of each batch row that are written, or queries of it that are there."""
    n, b = case["n"], case["batch"]
    most = n - int(case["ratio"] * n)
    if not case["ragged"] or case["n"] == 1:
        return [most] * b
    return [max(1, most - (i * most) // (4 * b)) for i in range(b)]


def _lengths(case):
    """Keys of each batch row, the new tokens' own among them."""
    b, held = case["batch"], case["held"]
    return [held - ((i * held) // (2 * b) if case["ragged"] else 0) for i in range(b)]


def _rows(case, heads, n, gen, spread):
    """[batch, heads, n, 128]: normal values, a few of each head's columns larger than the others."""
    out = torch.empty((case["batch"], heads, n, D), dtype=_type(case), device=DEVICE)
    gain = torch.exp(spread * torch.randn((heads, 1, D), generator=gen, device=DEVICE))
    for b in range(case["batch"]):
        out[b] = (torch.randn((heads, n, D), generator=gen, device=DEVICE) * gain).to(out.dtype)
    return out


def _by_token(x):
    """The same tensor, stored [batch][position][head][column]."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def _kept(case, gen):
    """Kept positions of each row, ascending, [batch, n] padded with -1."""
    b, n = case["batch"], case["n"]
    idx = torch.full((b, n), -1, dtype=torch.int32, device=DEVICE)
    for i, m in enumerate(_counts(case)):
        idx[i, :m] = torch.rand(n, generator=gen, device=DEVICE).argsort()[:m].sort().values.int()
    return idx


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    b, n, hq, hkv = case["batch"], case["n"], case["n_q_heads"], case["n_kv_heads"]
    x = {}
    if case["kind"] == "norm":
        x["q"], x["k"] = (_rows(case, h, n, gen, 0.5) for h in (hq, hkv))
        if case["by_token"]:
            x["q"], x["k"] = _by_token(x["q"]), _by_token(x["k"])
        x["wq"], x["wk"] = (1 + 0.2 * torch.randn(D, generator=gen, device=DEVICE) for _ in range(2))
        half = case["rot_dim"] // 2
        x["freq"] = torch.exp(torch.arange(half, dtype=torch.float64, device=DEVICE) * (-math.log(500000.0) / half))
        x["start"] = (case["first"] + torch.randint(0, 50, (b,), generator=gen, device=DEVICE)).int()
    elif case["kind"] == "store":
        x["k"], x["v"] = (_rows(case, hkv, n, gen, s) for s in (0.7, 0.2))
        x["idx"] = _kept(case, gen)
        x["count"] = torch.tensor(_counts(case), dtype=torch.int32, device=DEVICE)
        x["start"] = torch.full((b,), case["held"], dtype=torch.int32, device=DEVICE)
    else:
        x["q"] = _rows(case, hq, n, gen, 0.3)
        x["k"], x["v"] = (_rows(case, hkv, case["held"], gen, s) for s in (0.5, 0.2))
        x["count"] = torch.tensor(_counts(case), dtype=torch.int32, device=DEVICE)
        x["len"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)
    return x


# ------------------------------------------------------------------------------ plain form of the cache

def _quantise(x, bits):
    """x [..., 128] fp32 -> (codes of a value each, exponents of a block each), integers in int32."""
    blk = x.reshape(x.shape[:-1] + (D // BLOCK, BLOCK))
    # the smallest power of two s with max|x| <= 6 s (448 s): mantissas up to 1.5 (1.75) keep the exponent
    top = blk.abs().amax(-1).view(torch.int32)
    carry, back = (0x3FFFFF, 2) if bits == 4 else (0x1FFFFF, 8)
    exponent = (((top + carry) >> 23) - back).clamp(min=1)
    y = blk * ((254 - exponent) << 23).view(torch.float32)[..., None]          # x / s, exact
    if bits == 4:
        # to nearest, ties to the even code: values on a border go up where the code above is even
        a = y.abs()
        code = torch.zeros_like(a, dtype=torch.int32)
        for i, (border, up) in enumerate(((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                                          (3.5, True), (5.0, False))):
            code += (a >= border) if up else (a > border)
        code |= (y < 0).int() << 3
    else:
        code = y.to(torch.float8_e4m3fn).view(torch.uint8).int()
    return code.reshape(x.shape), exponent


def _values(code, exponent, bits):
    """The fp32 values that codes [..., 128] and exponents [..., 4] stand for."""
    if bits == 4:
        v = torch.tensor(FP4, device=code.device)[(code & 7).long()]
        v = torch.where(code >= 8, -v, v)
    else:
        v = code.to(torch.uint8).view(torch.float8_e4m3fn).float()
    s = (exponent.int() << 23).view(torch.float32)
    return (v.reshape(v.shape[:-1] + (D // BLOCK, BLOCK)) * s[..., None]).reshape(v.shape)


def _pack(code, exponent, bits, by_column):
    """Codes [..., rows, 128] and exponents [..., rows, 4] -> pages [..., rows / 64, bytes] (rows a multiple of 64)."""
    lead, pages = code.shape[:-2], code.shape[-2] // PAGE
    c = code.to(torch.uint8)
    if bits == 4:
        c = c[..., 0::2] | c[..., 1::2] << 4
    wide = c.shape[-1]
    e = exponent.to(torch.uint8)
    if not by_column:       # keys: rows as they are; scales [block][row % 16][row / 16]
        c = c.reshape(lead + (pages, PAGE * wide))
        e = e.reshape(lead + (pages, 4, 16, 4)).permute(*range(len(lead) + 1), -1, -2, -3)
    else:                   # values: [row / 4][column / 8][row % 4][eight columns]; scales [row / 4 % 4][block][row / 16][row % 4]
        c = c.reshape(lead + (pages, 16, 4, 16, wide // 16)).transpose(-2, -3)
        c = c.reshape(lead + (pages, PAGE * wide))
        e = e.reshape(lead + (pages, 4, 4, 4, 4)).permute(*range(len(lead) + 1), -3, -1, -4, -2)
    return torch.cat((c, e.reshape(lead + (pages, PAGE * 4))), -1).contiguous()


def _unpack(page, bits, by_column):
    """The inverse: codes [..., rows, 128] and exponents [..., rows, 4] in int32."""
    lead, pages, wide = page.shape[:-2], page.shape[-2], D * bits // 8
    c, e = page[..., :PAGE * wide], page[..., PAGE * wide:]
    if not by_column:
        e = e.reshape(lead + (pages, 4, 16, 4)).permute(*range(len(lead) + 1), -1, -2, -3)
    else:
        c = c.reshape(lead + (pages, 16, 16, 4, wide // 16)).transpose(-2, -3)
        e = e.reshape(lead + (pages, 4, 4, 4, 4)).permute(*range(len(lead) + 1), -2, -4, -1, -3)
    c = c.reshape(lead + (pages * PAGE, wide)).int()
    if bits == 4:
        c = torch.stack((c & 15, c >> 4), -1).reshape(lead + (pages * PAGE, D))
    return c, e.reshape(lead + (pages * PAGE, 4)).int()


# ------------------------------------------------------------------------------ what a program holds

class _State:
    """Inputs, and where the framework is called its handle, parameters, outputs and workspace."""


def prepare(case, seed):
    s = _State()
    s.case, x = case, _inputs(case, seed)
    b, n, hq, hkv = case["batch"], case["n"], case["n_q_heads"], case["n_kv_heads"]
    if case["kind"] == "attend":
        pages = (case["held"] + PAGE - 1) // PAGE
        for name, by_column in (("k", False), ("v", True)):
            raw, packed = x[name], []
            for row in range(b):     # (by rows: the fp32 copies of a long cache are large)
                padded = torch.zeros((hkv, pages * PAGE, D), device=DEVICE)
                padded[:, :case["held"]] = raw[row].float()
                packed.append(_pack(*_quantise(padded, case["bits"]), case["bits"], by_column))
            x[name] = torch.stack(packed)
            del raw, packed
    s.__dict__.update(x)
    if not own:
        return s
    from paper_2512_07090_amd import binding as B
    s.ctx = B.Context(0)
    strides = {}
    if case["by_token"]:
        strides = {"q_stride": s.q.stride()[:3], "kv_stride": s.k.stride()[:3], "o_stride": s.q.stride()[:3]}
    s.p = B.make_params((b, hq, n, D), (b, hkv, n, D), _type(case), 0.0, **strides)
    if case["kind"] == "norm":
        s.rot = B.make_rotary(s.freq, case["rot_dim"], q_weight=s.wq if case["norm"] else None,
                              k_weight=s.wk if case["norm"] else None, start=s.start, eps=EPS,
                              interleaved=case["interleaved"])
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
    elif case["kind"] == "store":
        s.cache = B.QuantCache(s.p, case["held"] + n, B.TF_CACHE_FP4 if case["bits"] == 4 else B.TF_CACHE_FP8, DEVICE)
        s.k_out, s.v_out = (torch.zeros_like(t) for t in (s.k, s.v))
    else:
        s.cache = B.QuantCache(s.p, case["held"], B.TF_CACHE_FP4 if case["bits"] == 4 else B.TF_CACHE_FP8, DEVICE)
        s.cache.k.copy_(s.k.reshape(-1))
        s.cache.v.copy_(s.v.reshape(-1))
        s.cache.len.copy_(s.len)
        s.k = s.v = None
        s.o = torch.empty_like(s.q)
        s.ws = torch.empty(B.tf_cache_workspace_bytes(s.p), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------------------ one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    kind = s.case["kind"]
    if kind == "norm":
        s.ctx.tf_norm_rotate(s.p, s.rot, s.q, s.k, s.q_out, s.k_out)
        return {"q": s.q_out, "k": s.k_out}
    if kind == "store":
        s.cache.len.copy_(s.start)             # back to where the rows are to go: the next request
        s.ctx.tf_cache_write(s.p, s.cache.desc, s.k, s.v, s.idx, s.case["n"], s.count)
        s.ctx.tf_cache_read(s.p, s.cache.desc, s.start, s.k_out, s.v_out)
        return {"k": s.k_out, "v": s.v_out, "len": s.cache.len}
    s.ctx.tf_cache_attend(s.p, s.cache.desc, s.q, s.o, s.count, s.ws)
    return {"o": s.o}


def _run_plain(s):
    case = s.case
    if case["kind"] == "norm":
        return {"q": _plain_norm(s, s.q, s.wq), "k": _plain_norm(s, s.k, s.wk)}
    if case["kind"] == "store":
        out = {}
        rows = s.idx.clamp(min=0).long()
        there = torch.arange(case["n"], device=DEVICE) < s.count[:, None]
        for name in ("k", "v"):
            x = getattr(s, name)
            y = torch.empty_like(x)
            for b in range(case["batch"]):
                v = _values(*_quantise(x[b][:, rows[b]].float(), case["bits"]), case["bits"])
                y[b] = torch.where(there[b][:, None], v, 0.0).to(x.dtype)
            out[name] = y
        out["len"] = s.start + s.count
        return out
    return {"o": _plain_attend(s)}


def _plain_norm(s, x, weight):
    case, y = s.case, x.float()
    if case["norm"]:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    pos = torch.arange(case["n"], device=DEVICE) + s.start[:, None].long()
    angle = pos.double()[..., None] * s.freq                                    # [batch, n, rot_dim / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = case["rot_dim"]
    turned, rest = y[..., :r], y[..., r:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if case["interleaved"] else (turned[..., :r // 2], turned[..., r // 2:])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((c, d), -1).flatten(-2) if case["interleaved"] else torch.cat((c, d), -1)
    return torch.cat((turned, rest), -1).to(x.dtype)


def _plain_attend(s):
    case = s.case
    b, n, hq, hkv, held = case["batch"], case["n"], case["n_q_heads"], case["n_kv_heads"], case["held"]
    key = torch.arange(held, device=DEVICE)
    t = torch.arange(n, device=DEVICE)
    o = torch.empty_like(s.q)
    for row in range(b):
        k = _values(*_unpack(s.k[row], case["bits"], False), case["bits"])[:, :held]
        v = _values(*_unpack(s.v[row], case["bits"], True), case["bits"])[:, :held]
        q = s.q[row].float().reshape(hkv, hq // hkv, n, D)
        # a query sees the keys up to its own; padding sees none and gets zeros
        sees = (key <= (s.len[row] - s.count[row] + t)[:, None]) & (t < s.count[row])[:, None]
        score = torch.matmul(q.reshape(hkv, -1, D), k.transpose(1, 2).contiguous()) / math.sqrt(D)
        score = score.reshape(hkv, hq // hkv, n, held).masked_fill(~sees, -math.inf)
        top = score.amax(-1, keepdim=True).clamp(min=-1e30)
        w = torch.exp(score - top)
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
        o[row] = torch.matmul(w.reshape(hkv, -1, held), v.contiguous()).reshape(hq, n, D).to(o.dtype)
    return o


# ------------------------------------------------------------------------------ the definition in 64 bits

def _grid(bits):
    """All magnitudes a code can stand for, ascending: the even ones in a tie are those at even places."""
    if bits == 4:
        g = [m / 2 for m in range(2)] + [2.0 ** e * (1 + m / 2) for e in range(3) for m in range(2)]
    else:
        g = [m / 8 * 2.0 ** -6 for m in range(8)] + [2.0 ** e * (1 + m / 8) for e in range(-6, 9) for m in range(8)][:-1]
    return torch.tensor(g, dtype=torch.float64, device=DEVICE)


def _rounded(x, bits):
    """x [..., 128] in 64 bits -> the values its quantised form stands for."""
    g = _grid(bits)
    blk = x.reshape(x.shape[:-1] + (D // BLOCK, BLOCK))
    top = blk.abs().amax(-1, keepdim=True) / g[-1]
    low = torch.tensor(-126.0, dtype=torch.float64, device=DEVICE)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -200)))
    e = torch.where(torch.exp2(e) < top, e + 1, e)        # whatever log2 did next to a power of two
    e = torch.where(torch.exp2(e - 1) >= top, e - 1, e)
    s = torch.exp2(torch.maximum(e, low))
    y = (blk / s).abs()
    hi = torch.searchsorted(g, y.contiguous()).clamp(max=len(g) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = g[hi] - y, y - g[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (torch.copysign(g[pick], blk) * s).reshape(x.shape)


def exact(case, seed):
    x = _inputs(case, seed)
    b, n, hq, hkv = case["batch"], case["n"], case["n_q_heads"], case["n_kv_heads"]
    if case["kind"] == "norm":
        out = {}
        r = case["rot_dim"]
        for name, w in (("q", x["wq"]), ("k", x["wk"])):
            y = x[name].double()
            if case["norm"]:
                y = y * torch.rsqrt(y.pow(2).sum(-1, keepdim=True) / D + EPS) * w.double()
            where = x["start"].double()[:, None] + torch.arange(n, dtype=torch.float64, device=DEVICE)
            turn = torch.polar(torch.ones((b, n, r // 2), dtype=torch.float64, device=DEVICE), where[..., None] * x["freq"])
            pair = y[..., :r].reshape(y.shape[:-1] + ((r // 2, 2) if case["interleaved"] else (2, r // 2)))
            if not case["interleaved"]:
                pair = pair.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
            if not case["interleaved"]:
                z = z.transpose(-1, -2)
            y = y.clone()
            y[..., :r] = z.reshape(y.shape[:-1] + (r,))
            out[name] = y
        return out
    if case["kind"] == "store":
        out = {}
        for name in ("k", "v"):
            y = torch.zeros((b, hkv, n, D), dtype=torch.float64, device=DEVICE)
            for row, m in enumerate(_counts(case)):
                y[row, :, :m] = _rounded(x[name][row][:, x["idx"][row, :m].long()].double(), case["bits"])
            out[name] = y
        out["len"] = None
        return out
    o = torch.zeros((b, hq, n, D), dtype=torch.float64, device=DEVICE)
    for row, (m, size) in enumerate(zip(_counts(case), _lengths(case))):
        for h in range(hkv):
            k, v = (_rounded(x[name][row, h, :size].double(), case["bits"]) for name in ("k", "v"))
            g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            score = x["q"][row, g, :m].double().reshape(-1, D) @ k.T.contiguous() * D ** -0.5
            future = torch.ones((m, size), dtype=torch.bool, device=DEVICE).triu(size - m + 1)
            score = score.reshape(-1, m, size).masked_fill(future, -math.inf)
            o[row, g, :m] = (torch.softmax(score, -1).reshape(-1, size) @ v).reshape(-1, m, D)
    return {"o": o}


# ------------------------------------------------------------------------------ what a pass needs

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    b, n, hq, hkv = case["batch"], case["n"], case["n_q_heads"], case["n_kv_heads"]
    row = D * case["bits"] / 8 + D / BLOCK                    # bytes of a quantised row
    if case["kind"] == "norm":
        values = b * n * (hq + hkv) * D
        return {"bytes": 2.0 * e * values, "flops": 8.0 * values}
    if case["kind"] == "store":
        rows = 2.0 * hkv * sum(_counts(case))
        return {"bytes": rows * (2 * D * e + row), "flops": 4.0 * rows * D}
    keys = sum(_lengths(case))
    pairs = sum(m * size - m * (m - 1) // 2 for m, size in zip(_counts(case), _lengths(case)))
    return {"bytes": 2.0 * hkv * keys * row + 2.0 * b * n * hq * D * e, "flops": 4.0 * D * hq * pairs}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (5e13 if case["dtype"] == "f32" else 5e14))
