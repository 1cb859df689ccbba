"""Cases of the operators around one attention block of a batched token step: paged K/V append with the position
rotation, attention of one new token over the paged cache, the gated and normalised residual between blocks, and
microscaled 4-bit rows (quantiser and product).

``run`` computes them in elementary torch operations (``own`` false) or through the library's entry points
(``own`` true); ``exact`` computes the same from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # one new token for each of 32 sequences of a 32-head model: what a serving step appends
        dict(name="append tokens", op="append", n_seq=32, new_min=1, new_max=1, past=2000, heads=32, kv_heads=32,
             head_dim=128, rotary=128, interleaved=False, page=16, dtype="bf16"),
        # several prompts written at once, ragged, on top of what the cache holds; keys and values shared by four heads
        dict(name="append prompts", op="append", n_seq=5, new_min=700, new_max=2900, past=300, heads=32, kv_heads=8,
             head_dim=128, rotary=128, interleaved=False, page=16, dtype="bf16"),
        # one sequence, a short context, four K/V heads of 64: the latency of a single user
        dict(name="attention one short", op="attention", n_seq=1, len_min=700, len_max=700, heads=32, kv_heads=4,
             head_dim=64, page=16, dtype="bf16"),
        # a serving batch of ragged lengths
        dict(name="attention ragged batch", op="attention", n_seq=64, len_min=1, len_max=4096, heads=32, kv_heads=8,
             head_dim=128, page=16, dtype="bf16"),
        # one long document: few rows, a long axis
        dict(name="attention long", op="attention", n_seq=1, len_min=131071, len_max=131071, heads=32, kv_heads=8,
             head_dim=128, page=64, dtype="bf16"),
        # the unquantised, unrounded form: fp32 caches, one K/V head per head, odd lengths
        dict(name="attention f32", op="attention", n_seq=7, len_min=1, len_max=1500, heads=8, kv_heads=8,
             head_dim=64, page=16, dtype="f32"),
        # the residual between two blocks for one token
        dict(name="norm glue token", op="glue", n_tok=1, d=4096, post=True, gate="row", pre=True, y="f32", dtype="bf16"),
        # the same over a long prompt
        dict(name="norm glue prompt", op="glue", n_tok=8191, d=5120, post=True, gate="full", pre=True, y="bf16",
             dtype="bf16"),
        # activations of a few tokens on their way into a 4-bit product
        dict(name="mx4 rows tokens", op="quantise", n_rows=33, d=2048, dtype="f32"),
        # a weight matrix, once when a model is loaded
        dict(name="mx4 rows weights", op="quantise", n_rows=11008, d=4096, dtype="bf16"),
        # one token through the vocabulary rows
        dict(name="mx4 product token", op="product", n_tok=1, n_rows=32000, d=4096, dtype="bf16"),
        # a prompt through one projection
        dict(name="mx4 product prompt", op="product", n_tok=4096, n_rows=11008, d=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "glue", "quantise", "product"])
    if op == "append":
        kv_heads = rng.choice([1, 2, 4, 8, 32])
        heads = 32 if kv_heads == 32 else kv_heads * rng.choice([1, 4, 5, 8])
        head_dim = rng.choice([64, 80, 128, 256])
        new = _log(rng, 1, 30_000_000 // ((heads + 2 * kv_heads) * head_dim))
        n_seq = rng.randint(1, min(new, 64))
        return dict(op=op, n_seq=n_seq, new_min=1, new_max=max(1, 2 * new // n_seq - 1), past=_log(rng, 1, 4000),
                    heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary=rng.choice([head_dim, head_dim // 2]),
                    interleaved=rng.random() < 0.5, page=rng.choice([16, 32, 64]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "attention":
        kv_heads = rng.choice([1, 2, 4, 8, 32])
        heads = kv_heads if kv_heads == 32 else kv_heads * rng.choice([1, 4, 5, 8, 16])
        head_dim = rng.choice([64, 80, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        room = (500_000_000 if dtype == "bf16" else 60_000_000) // (2 * kv_heads * head_dim * SIZE[dtype])
        total = _log(rng, 2, min(room, 131072))     # positions of all sequences
        n_seq = min(_log(rng, 1, 128), total)
        longest = max(1, 2 * total // n_seq - 1) if n_seq > 1 else total
        return dict(op=op, n_seq=n_seq, len_min=1 if n_seq > 1 else longest, len_max=longest, heads=heads,
                    kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]), dtype=dtype)
    if op == "glue":
        d = 8 * _log(rng, 16, 1024)
        return dict(op=op, n_tok=_log(rng, 1, 40_000_000 // d), d=d, post=rng.random() < 0.7,
                    gate=rng.choice(["none", "row", "full"]), pre=rng.random() < 0.7, y=rng.choice(["f32", "bf16"]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    d = 128 * _log(rng, 1, 64)
    if op == "quantise":
        return dict(op=op, n_rows=_log(rng, 1, 44_000_000 // d), d=d, dtype=rng.choice(["bf16", "f32"]))
    n_rows = _log(rng, 100, 11008 * 4096 // d if d > 1408 else 32000)
    return dict(op=op, n_tok=_log(rng, 1, 4096), n_rows=n_rows, d=d, dtype=rng.choice(["bf16", "bf16", "f32"]))


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, fixed by the case alone (a multiplicative hash of the index)."""
    if n == 1:
        return [hi]
    return [lo + ((i * 2654435761 + 97) % 4294967296) * (hi - lo + 1) // 4294967296 for i in range(n)]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 17)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _pages(g, lens, page):
    """A block table of pages in a shuffled order, and their number; the rows' unused entries name page 0."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 3, generator=g, device=DEV)[: sum(need)].to(torch.int32)
    table = torch.zeros((len(lens), max(max(need), 1)), dtype=torch.int32, device=DEV)
    cols = torch.arange(table.shape[1], device=DEV)
    table[cols[None] < torch.tensor(need, device=DEV)[:, None]] = order
    return table, sum(need) + 3


# ---- what a program has in hand ----------------------------------------------------------------------------------

def prepare(case, seed):
    return {"append": _prepare_append, "attention": _prepare_attention, "glue": _prepare_glue,
            "quantise": _prepare_quantise, "product": _prepare_product}[case["op"]](case, seed)


def _prepare_append(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    new = _spread(c["n_seq"], c["new_min"], c["new_max"])
    past = _spread(c["n_seq"], 0, c["past"])
    table, n_pages = _pages(g, [a + b for a, b in zip(new, past)], c["page"])
    n_tok, H, Hk, dh = sum(new), c["heads"], c["kv_heads"], c["head_dim"]
    counts = torch.tensor(new, device=DEV)
    seq = torch.repeat_interleave(torch.arange(c["n_seq"], device=DEV), counts)
    first = torch.cumsum(counts, 0) - counts
    pos = torch.arange(n_tok, device=DEV) - first[seq] + torch.tensor(past, device=DEV)[seq]
    qkv = _randn(g, (n_tok, H + 2 * Hk, dh), t)     # one projection's output: queries, keys and values side by side
    r = c["rotary"]
    return dict(case=c, q=qkv[:, :H], k=qkv[:, H:H + Hk], v=qkv[:, H + Hk:], pos=pos.to(torch.int32),
                seq=seq.to(torch.int32), table=table, n_pages=n_pages,
                inv_freq=10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r),
                K=_randn(g, (n_pages, Hk, c["page"], dh), t), V=_randn(g, (n_pages, Hk, c["page"], dh), t),
                q_out=torch.empty((n_tok, H, dh), dtype=t, device=DEV))


def _prepare_attention(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    lens = _spread(c["n_seq"], c["len_min"], c["len_max"])
    table, n_pages = _pages(g, lens, c["page"])
    shape = (n_pages, c["kv_heads"], c["page"], c["head_dim"])
    q = _randn(g, (c["n_seq"], c["heads"], c["head_dim"]), t)
    return dict(case=c, q=q, K=_randn(g, shape, t), V=_randn(g, shape, t), table=table, n_pages=n_pages,
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV), scale=c["head_dim"] ** -0.5,
                out=torch.empty_like(q), lse=torch.empty(q.shape[:2], dtype=torch.float32, device=DEV))


def _prepare_glue(c, seed):
    g, t, d, n = _gen(seed), TYPES[c["dtype"]], c["d"], c["n_tok"]
    gain = lambda: (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(t)  # noqa: E731
    gate = {"none": lambda: None, "row": lambda: torch.rand(d, generator=g, device=DEV).to(t),
            "full": lambda: torch.rand((n, d), generator=g, device=DEV).to(t)}[c["gate"]]()
    return dict(case=c, h=_randn(g, (n, d), torch.float32) * 3, y=_randn(g, (n, d), TYPES[c["y"]]),
                post=gain() if c["post"] else None, gate=gate, pre=gain() if c["pre"] else None, res=0.7, eps=1e-5,
                h_out=torch.empty((n, d), dtype=torch.float32, device=DEV), x_out=torch.empty((n, d), dtype=t, device=DEV))


def _scale_bytes(n_rows, d):
    return -(-n_rows // 128) * (d // 128) * 512


def _buffers(n_rows, d):
    return (torch.zeros((n_rows, d // 2), dtype=torch.uint8, device=DEV),
            torch.zeros(_scale_bytes(n_rows, d), dtype=torch.uint8, device=DEV))


def _prepare_quantise(c, seed):
    g, n, d, t = _gen(seed), c["n_rows"], c["d"], TYPES[c["dtype"]]
    Q, S = _buffers(n, d)
    return dict(case=c, W=(_randn(g, (n, d), torch.float32) * 0.02).to(t), Q=Q, S=S,
                out=torch.empty((n, d), dtype=t, device=DEV))


def _prepare_product(c, seed):
    g, n, d, t = _gen(seed), c["n_rows"], c["d"], TYPES[c["dtype"]]
    Qx, Sx = _buffers(c["n_tok"], d)
    codes, exps = _mx4_codes((_randn(g, (n, d), torch.float32) * 0.02).to(t))
    Qw, Sw = _mx4_pack(codes, exps)
    return dict(case=c, x=_randn(g, (c["n_tok"], d), t), Qx=Qx, Sx=Sx, Qw=Qw, Sw=Sw,
                out=torch.empty((c["n_tok"], n), dtype=t, device=DEV))


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attention": _plain_attention, "glue": _plain_glue, "quantise": _plain_quantise,
            "product": _plain_product}[s["case"]["op"]](s)


def _own(s):
    from paper_2601_11676_b200 import binding as B
    c = s["case"]
    code = B.F32 if c["dtype"] == "f32" else B.BF16
    op = c["op"]
    if op in ("append", "attention") and "shape" not in s:
        s["shape"] = B.paged_shape(c["heads"], c["kv_heads"], c["head_dim"], c["page"], s["n_pages"],
                                   s["table"].shape[1], code)
    if op == "append":
        B.halo_paged_kv_append(s["shape"], s["q"], s["k"], s["v"], s["pos"], s["seq"], s["table"], s["inv_freq"],
                               c["interleaved"], s["q_out"], s["K"], s["V"])
        return s["q_out"], s["K"], s["V"]
    if op == "attention":
        if "ws" not in s:
            s["ws"] = torch.empty(B.halo_paged_mha_workspace_bytes(s["shape"], c["n_seq"]), dtype=torch.uint8, device=DEV)
        B.halo_paged_mha(s["shape"], s["q"], s["K"], s["V"], s["table"], s["lens"], s["scale"], s["out"], s["ws"],
                         lse=s["lse"])
        return s["out"], s["lse"]
    if op == "glue":
        if "shape" not in s:
            s["shape"] = B.norm_shape(c["d"], s["eps"], B.F32 if c["y"] == "f32" else B.BF16, code)
        B.halo_norm_glue(s["shape"], s["h"], s["y"], s["post"], s["gate"], s["res"], s["pre"], s["h_out"], s["x_out"])
        return s["h_out"], s["x_out"]
    if op == "quantise":
        B.halo_quantize_rows_mx4(c["d"], c["n_rows"], code, s["W"], s["Q"], s["S"])
        B.halo_dequantize_rows_mx4(c["d"], c["n_rows"], code, s["Q"], s["S"], s["out"])
        return s["out"]
    B.halo_quantize_rows_mx4(c["d"], c["n_tok"], code, s["x"], s["Qx"], s["Sx"])
    B.halo_product_mx4(c["d"], c["n_tok"], c["n_rows"], s["Qx"], s["Sx"], s["Qw"], s["Sw"], code, s["out"])
    return s["out"]


def _turn(x, cos, sin, r, interleaved):
    """Rotates the first r elements of the last axis, pairs (2i, 2i+1) or (i, i + r/2); fp32."""
    x = x.float()
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)
    a, b = x[..., : r // 2], x[..., r // 2:r]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)


def _plain_append(s):
    c, t = s["case"], s["K"].dtype
    angle = s["pos"].double()[:, None] * s["inv_freq"]          # far positions lose their angle in 32 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    q = _turn(s["q"], cos, sin, c["rotary"], c["interleaved"]).to(t)
    k = _turn(s["k"], cos, sin, c["rotary"], c["interleaved"]).to(t)
    pos = s["pos"].long()
    page, at = s["table"][s["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    s["K"][page, :, at] = k
    s["V"][page, :, at] = s["v"]
    return q, s["K"], s["V"]


def _plain_attention(s):
    c, q = s["case"], s["q"]
    n, Hk, dh = c["n_seq"], c["kv_heads"], c["head_dim"]
    K = s["K"][s["table"].long()].float().transpose(1, 2).reshape(n, Hk, -1, dh)
    V = s["V"][s["table"].long()].float().transpose(1, 2).reshape(n, Hk, -1, dh)
    scores = torch.matmul(q.float().view(n, Hk, -1, dh), K.transpose(-1, -2)) * s["scale"]
    there = torch.arange(K.shape[2], device=q.device)[None] < s["lens"][:, None]
    scores = scores.masked_fill(~there[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)     # a sequence of no positions gives zeros
    p = torch.exp(scores - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, V) / torch.where(l == 0, torch.ones_like(l), l)
    return o.reshape(q.shape).to(q.dtype), (m + torch.log(l)).reshape(n, c["heads"])


def _plain_glue(s):
    y = s["y"].float()
    if s["post"] is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * s["post"].float()
    if s["gate"] is not None:
        y = y * s["gate"].float()
    h = s["h"] + s["res"] * y
    x = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"])
    if s["pre"] is not None:
        x = x * s["pre"].float()
    return h, x.to(s["x_out"].dtype)


def _mx4_codes(W):
    """Codes 0..15 (sign, 2 exponent bits, 1 mantissa bit) [n][d] and exponents [n][d/32] of the blocks of 32."""
    w = W.float().view(W.shape[0], -1, 32)
    amax = w.abs().amax(-1)
    exps = torch.where(amax > 0, torch.frexp(amax).exponent - 3, torch.full_like(amax, -127).int()).clamp(min=-127)
    a = torch.ldexp(w.abs().double(), -exps[..., None]).float()     # below 8; 2^127 is past fp32's ldexp
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    v = (torch.round(a / step) * step).clamp(max=6)                 # ties to the even code
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    code = code + 8 * torch.signbit(w).to(torch.uint8)
    return code.view(W.shape), exps


def _mx4_pack(code, exps):
    """Two codes a byte, the lower element in the low half; scales (exponent + 127) in blocks of 128 rows x 4."""
    Q = code[:, 0::2] | (code[:, 1::2] << 4)
    n, nb = exps.shape
    tiles = -(-n // 128)
    S = torch.zeros((tiles * 128, nb), dtype=torch.uint8, device=exps.device)
    S[:n] = (exps + 127).to(torch.uint8)
    return Q, S.view(tiles, 4, 32, nb // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _mx4_values(code, exps):
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    v = table[code.long()].view(code.shape[0], -1, 32)
    return torch.ldexp(v.double(), exps[..., None]).float().view(code.shape)


def _mx4_unpack(Q, S, n, d):
    code = torch.stack([Q & 15, Q >> 4], -1).view(n, d)
    exps = S.view(-1, d // 128, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, d // 32)[:n].int() - 127
    return code, exps


def _plain_quantise(s):
    return _mx4_values(*_mx4_codes(s["W"])).to(s["W"].dtype)


def _plain_product(s):
    c = s["case"]
    x = _mx4_values(*_mx4_codes(s["x"]))
    w = _mx4_values(*_mx4_unpack(s["Qw"], s["Sw"], c["n_rows"], c["d"]))
    return torch.matmul(x, w.t()).to(s["x"].dtype)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["op"] == "append":
        n = sum(_spread(c["n_seq"], c["new_min"], c["new_max"]))
        return dict(bytes=2 * n * (c["heads"] + 2 * c["kv_heads"]) * c["head_dim"] * e + n * 12,
                    flops=3 * n * (c["heads"] + c["kv_heads"]) * c["rotary"])
    if c["op"] == "attention":
        n = sum(_spread(c["n_seq"], c["len_min"], c["len_max"]))
        rows = c["n_seq"] * c["heads"]
        return dict(bytes=2 * n * c["kv_heads"] * c["head_dim"] * e + 2 * rows * c["head_dim"] * e + 4 * rows,
                    flops=4 * n * c["heads"] * c["head_dim"])
    if c["op"] == "glue":
        cells = c["n_tok"] * c["d"]
        gate = {"none": 0, "row": c["d"], "full": cells}[c["gate"]]
        return dict(bytes=cells * (8 + SIZE[c["y"]] + e) + (gate + c["d"] * (c["post"] + c["pre"])) * e, flops=8 * cells)
    if c["op"] == "quantise":       # the rows in, codes and scales out; codes and scales in, the values out
        cells = c["n_rows"] * c["d"]
        return dict(bytes=2 * cells * e + 2 * (cells // 2 + cells // 32), flops=4 * cells)
    x, w, y = c["n_tok"] * c["d"], c["n_rows"] * c["d"], c["n_tok"] * c["n_rows"]
    return dict(bytes=x * e + w // 2 + w // 32 + y * e, flops=2 * c["n_tok"] * w)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "glue": _exact_glue, "quantise": _exact_quantise,
            "product": _exact_product}[case["op"]](case, s)


def _exact_append(c, s):
    r, dh = c["rotary"], c["head_dim"]
    first = torch.arange(0, r, 2, device=DEV) if c["interleaved"] else torch.arange(r // 2, device=DEV)
    other = first + (1 if c["interleaved"] else r // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None, None] * s["inv_freq"])

    def rotated(x):
        x = x.double().clone()
        z = torch.complex(x[..., first], x[..., other]) * turn
        x[..., first], x[..., other] = z.real, z.imag
        return x

    K, V = s["K"].double(), s["V"].double()
    flat = (s["table"][s["seq"].long(), s["pos"].long() // c["page"]].long(), s["pos"].long() % c["page"])
    heads = torch.arange(c["kv_heads"], device=DEV)
    K.index_put_((flat[0][:, None], heads[None], flat[1][:, None]), rotated(s["k"]))
    V.index_put_((flat[0][:, None], heads[None], flat[1][:, None]), s["v"].double())
    assert K.shape[-1] == dh
    return rotated(s["q"]), K, V


def _exact_attention(c, s):
    n, H, Hk, dh, page = c["n_seq"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    out = torch.zeros((n, H, dh), dtype=torch.float64, device=DEV)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64, device=DEV)
    for i, length in enumerate(s["lens"].tolist()):
        if length == 0:
            continue
        pages = s["table"][i, : -(-length // page)].long()
        for h in range(Hk):
            K = s["K"][pages, h].reshape(-1, dh)[:length].double()
            V = s["V"][pages, h].reshape(-1, dh)[:length].double()
            rows = slice(h * (H // Hk), (h + 1) * (H // Hk))
            score = s["q"][i, rows].double() @ K.t() * s["scale"]
            lse[i, rows] = torch.logsumexp(score, -1)
            out[i, rows] = torch.softmax(score, -1) @ V
    return out, lse


def _exact_glue(c, s):
    one = torch.ones((), dtype=torch.float64, device=DEV)
    post, gate, pre = (one if s[k] is None else s[k].double() for k in ("post", "gate", "pre"))
    y = s["y"].double()
    if s["post"] is not None:
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / c["d"] + s["eps"])
    h = s["h"].double() + s["res"] * (gate * (post * y))
    return h, pre * (h / torch.sqrt(h.square().sum(-1, keepdim=True) / c["d"] + s["eps"]))


def _exact_values(W):
    """The nearest of the sixteen values times the block's power of two, by borders between neighbouring values."""
    w = W.double().view(W.shape[0], -1, 32)
    top = w.abs().amax(-1, keepdim=True)
    unit = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2),
                       torch.ones_like(top))
    unit = torch.where(top >= unit * 8, unit * 2, torch.where(top < unit * 4, unit / 2, unit)).clamp(min=2.0 ** -127)
    unit = torch.where(top > 0, unit, torch.ones_like(unit))
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    # at a border the value with the even code wins: the codes 0, 2, 4, 6 keep the border above and below them
    a, best = w.abs() / unit, torch.zeros_like(w)
    for i in range(7):
        border = (grid[i] + grid[i + 1]) / 2
        best = torch.where((a >= border) if i % 2 else (a > border), grid[i + 1], best)
    return (torch.copysign(best, w) * unit).view(W.shape)


def _exact_quantise(c, s):
    return _exact_values(s["W"])


def _exact_product(c, s):
    n, d = c["n_rows"], c["d"]
    low, high = (s["Qw"] & 15).long(), (s["Qw"] >> 4).long()
    code = torch.empty((n, d), dtype=torch.long, device=DEV)
    code[:, 0::2], code[:, 1::2] = low, high
    size = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)[code & 7]
    row, block = torch.arange(n, device=DEV)[:, None], torch.arange(d // 32, device=DEV)[None]
    where = ((row // 128) * (d // 128) + block // 4) * 512 + (row % 32) * 16 + (row % 128 // 32) * 4 + block % 4
    unit = torch.exp2(s["Sw"][where].double() - 127).repeat_interleave(32, 1)
    return _exact_values(s["x"]) @ (torch.where(code > 7, -size, size) * unit).t()
