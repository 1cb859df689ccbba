"""Cases of the operators around a paged cache that holds prompts and 8-bit rows: the append that norms queries and keys
per head and turns them, the 8-bit rows it writes and their way back, attention of one new token over 8-bit rows, and
causal attention of packed chunks of new tokens.

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
        # one new token for each of 32 sequences, into an 8-bit cache: what a serving step appends (and reads back here, so
        # that the values behind the codes are compared)
        dict(name="append tokens", op="append", n_seq=32, new_min=1, new_max=1, past=2000, heads=32, kv_heads=8, head_dim=128,
             rotary=128, interleaved=False, turn_scale=1.0, norm="both", page=16, eight=True, dtype="bf16"),
        # several prompts written at once, ragged, on top of what the 8-bit cache holds; frequencies stretched for a long context
        dict(name="append prompts", op="append", n_seq=5, new_min=700, new_max=2900, past=300, heads=32, kv_heads=8,
             head_dim=128, rotary=128, interleaved=False, turn_scale=1.1386, norm="both", page=16, eight=True, dtype="bf16"),
        # unrounded caches, pairs side by side, half the head turned
        dict(name="append f32", op="append", n_seq=7, new_min=1, new_max=400, past=500, heads=8, kv_heads=8, head_dim=64,
             rotary=32, interleaved=True, turn_scale=1.0, norm="both", page=16, eight=False, dtype="f32"),
        # one sequence, a short context, four K/V heads of 64: the latency of a single user
        dict(name="8-bit one short", op="token", n_seq=1, len_min=700, len_max=700, heads=32, kv_heads=4, head_dim=64, page=16),
        # a serving batch of ragged lengths
        dict(name="8-bit ragged batch", op="token", n_seq=64, len_min=1, len_max=4096, heads=32, kv_heads=8, head_dim=128,
             page=16),
        # one long document: few rows, a long axis
        dict(name="8-bit long", op="token", n_seq=1, len_min=131071, len_max=131071, heads=32, kv_heads=8, head_dim=128, page=64),
        # a prompt of a single user, nothing cached before it
        dict(name="prompt", op="chunk", n_seq=1, new_min=4096, new_max=4096, past_min=0, past_max=0, heads=32, kv_heads=8,
             head_dim=128, page=16, eight=False, dtype="bf16"),
        # prompts of several users packed, some behind a cached prefix; one K/V head per head
        dict(name="packed prompts", op="chunk", n_seq=7, new_min=1, new_max=1500, past_min=0, past_max=1201, heads=32,
             kv_heads=32, head_dim=128, page=32, eight=False, dtype="bf16"),
        # a chunk of a long prompt over what is cached of it in 8 bits
        dict(name="chunk 8-bit long", op="chunk", n_seq=1, new_min=512, new_max=512, past_min=32000, past_max=32000, heads=32,
             kv_heads=8, head_dim=128, page=64, eight=True, dtype="bf16"),
        # a few drafted tokens for each sequence of a batch
        dict(name="drafted tokens", op="chunk", n_seq=16, new_min=1, new_max=8, past_min=5, past_max=4000, heads=32, kv_heads=8,
             head_dim=128, page=16, eight=False, dtype="bf16"),
        # wide heads, an odd chunk
        dict(name="wide heads", op="chunk", n_seq=2, new_min=333, new_max=1000, past_min=0, past_max=1001, heads=16, kv_heads=2,
             head_dim=256, page=16, eight=False, dtype="bf16"),
        # the unrounded form: fp32 caches, odd lengths
        dict(name="chunk f32", op="chunk", n_seq=3, new_min=1, new_max=300, past_min=0, past_max=400, heads=8, kv_heads=8,
             head_dim=64, page=16, eight=False, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "token", "chunk", "chunk"])
    kv_heads = rng.choice([1, 2, 4, 8, 32])
    heads = kv_heads if kv_heads == 32 else kv_heads * rng.choice([1, 4, 5, 8, 16] if op == "token" else [1, 4, 5, 8])
    head_dim = rng.choice([64, 80, 128, 256])
    page = rng.choice([16, 32, 64])
    if op == "append":
        new = _log(rng, 1, 30_000_000 // ((heads + 2 * kv_heads) * head_dim))
        n_seq = rng.randint(1, min(new, 64))
        eight = rng.random() < 0.6
        return dict(op=op, n_seq=n_seq, new_min=1, new_max=max(1, 2 * new // n_seq - 1), past=_log(rng, 1, 4000),
                    heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary=rng.choice([head_dim, head_dim // 2]),
                    interleaved=rng.random() < 0.5, turn_scale=rng.choice([1.0, 1.25]),
                    norm=rng.choice(["both", "both", "keys", "none"]), page=page, eight=eight,
                    dtype="bf16" if eight else rng.choice(["bf16", "f32"]))
    if op == "token":
        total = _log(rng, 2, min(250_000_000 // (2 * kv_heads * head_dim), 131072))     # positions of all sequences
        n_seq = min(_log(rng, 1, 128), total)
        longest = max(1, 2 * total // n_seq - 1) if n_seq > 1 else total
        return dict(op=op, n_seq=n_seq, len_min=1 if n_seq > 1 else longest, len_max=longest, heads=heads,
                    kv_heads=kv_heads, head_dim=head_dim, page=page)
    eight = rng.random() < 0.3
    dtype = "bf16" if eight else rng.choice(["bf16", "bf16", "bf16", "f32"])
    # rows of all sequences as if each were the longest, times the longest length: bounds the work and the padded plain form
    cells = (400_000_000 if dtype == "bf16" else 20_000_000) // heads
    n_seq = _log(rng, 1, 32)
    new = _log(rng, 1, max(1, min(4096, math.isqrt(cells // n_seq))))
    past = _log(rng, 1, max(1, min(32000, cells // (n_seq * new) - new)))
    return dict(op=op, n_seq=n_seq, new_min=1 if n_seq > 1 else new, new_max=new, past_min=0, past_max=past, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, page=page, eight=eight, dtype=dtype)


def _spread(n, lo, hi, salt=97):
    """n whole numbers from lo to hi, fixed by the case alone (a multiplicative hash of the index)."""
    if n == 1:
        return [hi]
    return [lo + ((i * 2654435761 + salt) % 4294967296) * (hi - lo + 1) // 4294967296 for i in range(n)]


def _counts(c):
    """New tokens and cached positions in front of them, per sequence."""
    if c["op"] == "append":
        return _spread(c["n_seq"], c["new_min"], c["new_max"]), _spread(c["n_seq"], 0, c["past"])
    return _spread(c["n_seq"], c["new_min"], c["new_max"]), _spread(c["n_seq"], c["past_min"], c["past_max"], 1234567891)


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


def _cache(g, c, n_pages):
    """Keys and values of a cache that is in use: codes and scale bytes of 8-bit rows, or rows in the case's type."""
    shape = (n_pages, c["kv_heads"], c["page"], c["head_dim"])
    if not c.get("eight", True):
        t = TYPES[c["dtype"]]
        return dict(K=_randn(g, shape, t), V=_randn(g, shape, t), Ks=None, Vs=None)
    K, Ks = _to_eight(_randn(g, shape, torch.bfloat16))
    V, Vs = _to_eight(_randn(g, shape, torch.bfloat16) * 3)
    return dict(K=K, V=V, Ks=Ks, Vs=Vs)


# ---- what a program has in hand ----------------------------------------------------------------------------------

def prepare(case, seed):
    return {"append": _prepare_append, "token": _prepare_token, "chunk": _prepare_chunk}[case["op"]](case, seed)


def _prepare_append(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    new, past = _counts(c)
    table, n_pages = _pages(g, [a + b for a, b in zip(new, past)], c["page"])
    n_tok, H, Hk, dh, r = sum(new), c["heads"], c["kv_heads"], c["head_dim"], c["rotary"]
    counts = torch.tensor(new, device=DEV)
    seq = torch.repeat_interleave(torch.arange(c["n_seq"], device=DEV), counts)
    first = torch.cumsum(counts, 0) - counts
    pos = torch.arange(n_tok, device=DEV) - first[seq] + torch.tensor(past, device=DEV)[seq]
    qkv = _randn(g, (n_tok, H + 2 * Hk, dh), t)     # one projection's output: queries, keys and values side by side
    gain = lambda: (1 + 0.2 * torch.randn(dh, generator=g, device=DEV)).to(t)  # noqa: E731
    w_q, w_k = gain(), gain()
    row = lambda: torch.empty((n_tok, Hk, dh), dtype=t, device=DEV)  # noqa: E731
    return dict(case=c, q=qkv[:, :H], k=qkv[:, H:H + Hk], v=qkv[:, H + Hk:], pos=pos.to(torch.int32), seq=seq.to(torch.int32),
                table=table, n_pages=n_pages, w_q=w_q if c["norm"] == "both" else None,
                w_k=w_k if c["norm"] != "none" else None, eps=1e-6,
                inv_freq=10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r),
                q_out=torch.empty((n_tok, H, dh), dtype=t, device=DEV), k_out=row(), v_out=row(), **_cache(g, c, n_pages))


def _prepare_token(c, seed):
    g = _gen(seed)
    lens = _spread(c["n_seq"], c["len_min"], c["len_max"])
    table, n_pages = _pages(g, lens, c["page"])
    q = _randn(g, (c["n_seq"], c["heads"], c["head_dim"]), torch.bfloat16)
    return dict(case=c, q=q, table=table, n_pages=n_pages, lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                scale=c["head_dim"] ** -0.5, out=torch.empty_like(q),
                lse=torch.empty(q.shape[:2], dtype=torch.float32, device=DEV), **_cache(g, c, n_pages))


def _prepare_chunk(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    new, past = _counts(c)
    lens = [a + b for a, b in zip(new, past)]
    table, n_pages = _pages(g, lens, c["page"])
    q = _randn(g, (sum(new), c["heads"], c["head_dim"]), t)
    start = torch.zeros(c["n_seq"] + 1, dtype=torch.int32, device=DEV)
    start[1:] = torch.cumsum(torch.tensor(new, device=DEV), 0)
    return dict(case=c, q=q, start=start, table=table, n_pages=n_pages, max_new=max(new),
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV), scale=c["head_dim"] ** -0.5, out=torch.empty_like(q),
                lse=torch.empty(q.shape[:2], dtype=torch.float32, device=DEV), **_cache(g, c, n_pages))


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "token": _plain_token, "chunk": _plain_chunk}[s["case"]["op"]](s)


def _own(s):
    from paper_2601_11676_b200 import binding as B
    c, op = s["case"], s["case"]["op"]
    if "shape" not in s:
        code = B.F32 if c.get("dtype") == "f32" else B.BF16
        s["shape"] = B.paged_shape(c["heads"], c["kv_heads"], c["head_dim"], c["page"], s["n_pages"], s["table"].shape[1], code)
        need = B.halo_paged_mha_f8_workspace_bytes(s["shape"], c["n_seq"]) if op == "token" else \
            B.halo_paged_prompt_mha_workspace_bytes(s["shape"], s["q"].shape[0], c["n_seq"]) if op == "chunk" else 0
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    if op == "append":
        B.halo_paged_norm_append(s["shape"], s["q"], s["k"], s["v"], s["w_q"], s["w_k"], s["eps"], s["pos"], s["seq"],
                                 s["table"], s["inv_freq"], c["interleaved"], c["turn_scale"], s["q_out"], s["K"], s["V"],
                                 s["Ks"], s["Vs"])
        if not c["eight"]:
            return s["q_out"], s["K"], s["V"]
        B.halo_paged_kv_read(s["shape"], s["pos"], s["seq"], s["table"], s["K"], s["V"], s["k_out"], s["v_out"], s["Ks"], s["Vs"])
        return s["q_out"], s["k_out"], s["v_out"]
    if op == "token":
        B.halo_paged_mha_f8(s["shape"], s["q"], s["K"], s["V"], s["Ks"], s["Vs"], s["table"], s["lens"], s["scale"], s["out"],
                            s["ws"], lse=s["lse"])
    else:
        B.halo_paged_prompt_mha(s["shape"], s["q"], s["start"], s["K"], s["V"], s["table"], s["lens"], s["scale"], s["out"],
                                s["ws"], s["Ks"], s["Vs"], lse=s["lse"])
    return s["out"], s["lse"]


def _to_eight(x):
    """Codes (bytes) of rows of the last axis and their scale bytes: e + 127, e the smallest whole number with
    amax <= 448 * 2^e; a code is the nearest e4m3 number of x * 2^-e."""
    x = x.float()
    f, up = torch.frexp(x.abs().amax(-1))
    e = torch.where(f > 0, up - torch.where(f <= 0.875, 9, 8), -117).clamp(-117, 119)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _from_eight(codes, scales):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), scales.int()[..., None] - 127)


def _turn(x, cos, sin, r, interleaved):
    """Rotates the first r elements of the last axis, pairs (2i, 2i+1) or (i, i + r/2); fp32."""
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)
    a, b = x[..., : r // 2], x[..., r // 2:r]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)


def _plain_append(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["inv_freq"]          # far positions lose their angle in 32 bits
    cos, sin = ((f(angle) * c["turn_scale"]).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w.float()
        return _turn(x, cos, sin, c["rotary"], c["interleaved"])

    q, k = turned(s["q"], s["w_q"]).to(s["q"].dtype), turned(s["k"], s["w_k"])
    pos = s["pos"].long()
    page, at = s["table"][s["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    if not c["eight"]:
        s["K"][page, :, at] = k.to(s["K"].dtype)
        s["V"][page, :, at] = s["v"]
        return q, s["K"], s["V"]
    s["K"][page, :, at], s["Ks"][page, :, at] = _to_eight(k)
    s["V"][page, :, at], s["Vs"][page, :, at] = _to_eight(s["v"])
    back = lambda codes, scales: _from_eight(codes[page, :, at], scales[page, :, at]).to(q.dtype)  # noqa: E731
    return q, back(s["K"], s["Ks"]), back(s["V"], s["Vs"])


def _rows_of(s, codes, scales):
    """The cache's rows by sequence, K/V head and position, in fp32."""
    c, at = s["case"], s["table"].long()
    x = codes[at].float() if scales is None else _from_eight(codes[at], scales[at])
    return x.transpose(1, 2).reshape(c["n_seq"], c["kv_heads"], -1, c["head_dim"])


def _attend(s, q, seen):
    """q [n_seq][heads][rows][head_dim], fp32; seen: positions that a row of a sequence sees [n_seq][rows]."""
    c = s["case"]
    K, V = _rows_of(s, s["K"], s["Ks"]), _rows_of(s, s["V"], s["Vs"])
    q = q.reshape(c["n_seq"], c["kv_heads"], -1, q.shape[-1])          # the rows of all heads that share keys
    scores = torch.matmul(q, K.transpose(-1, -2)).view(c["n_seq"], c["heads"], -1, K.shape[2]) * s["scale"]
    there = torch.arange(K.shape[2], device=q.device) < seen[:, None, :, None]
    scores = scores.masked_fill_(~there, -math.inf)
    m = scores.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)     # a row that sees nothing gives zeros
    p = scores.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(c["n_seq"], c["kv_heads"], -1, K.shape[2]), V).view(*p.shape[:3], -1)
    return o / torch.where(l == 0, torch.ones_like(l), l), (m + torch.log(l))[..., 0]


def _plain_token(s):
    out, lse = _attend(s, s["q"].float()[:, :, None], s["lens"][:, None])
    return out[:, :, 0].to(s["q"].dtype), lse[..., 0]


def _plain_chunk(s):
    q, start, lens = s["q"], s["start"].long(), s["lens"].long()
    new = start[1:] - start[:-1]
    row = torch.arange(s["max_new"], device=q.device)
    there = row < new[:, None]                                          # sequences padded to the longest chunk
    padded = torch.zeros((len(lens), s["max_new"], *q.shape[1:]), device=q.device)
    padded[there] = q.float()
    out, lse = _attend(s, padded.transpose(1, 2), (lens - new)[:, None] + row + 1)
    return out.transpose(1, 2)[there].to(q.dtype), lse.transpose(1, 2)[there]


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c = case
    H, Hk, dh = c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        n, e = sum(_counts(c)[0]), SIZE[c["dtype"]]
        # the rows in and out; 8 bits: codes and scales out, in again, and the values out
        cache = 2 * Hk * ((2 * (dh + 1) + dh * e) if c["eight"] else dh * e)
        return dict(bytes=n * ((H + 2 * Hk) * dh * e + H * dh * e + cache + 12),
                    flops=n * (H + Hk) * (3 * c["rotary"] + 4 * dh))
    if c["op"] == "token":
        n, rows = sum(_spread(c["n_seq"], c["len_min"], c["len_max"])), c["n_seq"] * H
        return dict(bytes=2 * n * Hk * (dh + 1) + 4 * rows * dh + 4 * rows, flops=4 * n * H * dh)
    new, past = _counts(c)
    e, rows = SIZE[c["dtype"]], sum(new) * H
    row = dh + 1 if c["eight"] else dh * e
    return dict(bytes=2 * (sum(new) + sum(past)) * Hk * row + 2 * rows * dh * e + 4 * rows,
                flops=4 * H * dh * sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past)))


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "token": _exact_token, "chunk": _exact_chunk}[case["op"]](case, s)


def _exact_eight(x):
    """The values that 8-bit rows of x stand for, by the spacing of the numbers with 3 bits behind the point."""
    top = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448)))
    unit = torch.where(unit * 448 < top, unit * 2, torch.where(unit * 224 >= top, unit / 2, unit))
    unit = torch.where(top > 0, unit, torch.ones_like(unit)).clamp(2.0 ** -117, 2.0 ** 119)
    a = (x / unit).abs()
    octave = torch.floor(torch.log2(torch.where(a > 0, a, torch.ones_like(a)))).clamp(min=-6)
    gap = torch.exp2(octave - 3)
    return torch.copysign(torch.round(a / gap) * gap, x) * unit         # round(): ties to even


def _exact_append(c, s):
    r = c["rotary"]
    first = torch.arange(0, r, 2, device=DEV) if c["interleaved"] else torch.arange(r // 2, device=DEV)
    other = first + (1 if c["interleaved"] else r // 2)
    length = torch.full((), c["turn_scale"], dtype=torch.float64, device=DEV)
    turn = torch.polar(length, s["pos"].double()[:, None, None] * s["inv_freq"])

    def turned(x, w):
        x = x.double().clone()
        if w is not None:
            x = w.double() * (x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["head_dim"] + s["eps"]))
        z = torch.complex(x[..., first], x[..., other]) * turn
        x[..., first], x[..., other] = z.real, z.imag
        return x

    q, k, v = turned(s["q"], s["w_q"]), turned(s["k"], s["w_k"]), s["v"].double()
    if c["eight"]:
        return q, _exact_eight(k), _exact_eight(v)
    K, V = s["K"].double(), s["V"].double()
    flat = (s["table"][s["seq"].long(), s["pos"].long() // c["page"]].long(), s["pos"].long() % c["page"])
    heads = torch.arange(c["kv_heads"], device=DEV)
    K.index_put_((flat[0][:, None], heads[None], flat[1][:, None]), k)
    V.index_put_((flat[0][:, None], heads[None], flat[1][:, None]), v)
    return q, K, V


def _exact_values(codes, scales):
    """Codes: a sign, four bits of exponent, three behind the point."""
    if scales is None:
        return codes.double()
    code = codes.int()
    up, part = (code >> 3) & 15, (code & 7).double()
    size = torch.where(up > 0, (1 + part / 8) * torch.exp2(up.double() - 7), part * 2.0 ** -9)
    return torch.where(code > 127, -size, size) * torch.exp2(scales.double() - 127)[..., None]


def _exact_rows(c, s, seq, first, out, lse):
    """Rows of sequence `seq` into out[rows][heads][head_dim] and lse[rows][heads]; row i sees first + i positions."""
    n, length, G = out.shape[0], int(s["lens"][seq]), c["heads"] // c["kv_heads"]
    q = s["q"][seq:seq + 1] if c["op"] == "token" else s["q"][int(s["start"][seq]):int(s["start"][seq + 1])]
    pages = s["table"][seq, : -(-length // c["page"])].long()
    hidden = torch.arange(length, device=DEV)[None] >= first + torch.arange(n, device=DEV)[:, None]
    for h in range(c["heads"]):
        kv = h // G
        K, V = (_exact_values(s[k][pages, kv], None if s[k + "s"] is None else s[k + "s"][pages, kv])
                .reshape(-1, c["head_dim"])[:length] for k in ("K", "V"))
        score = (q[:, h].double() @ K.t() * s["scale"]).masked_fill(hidden, -math.inf)
        lse[:, h] = torch.logsumexp(score, -1)
        out[:, h] = torch.softmax(score, -1) @ V


def _exact_token(c, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for i, length in enumerate(s["lens"].tolist()):
        if length > 0:
            _exact_rows(c, s, i, length, out[i:i + 1], lse[i:i + 1])
    return out, lse


def _exact_chunk(c, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    start = s["start"].tolist()
    for i, length in enumerate(s["lens"].tolist()):
        a, b = start[i], start[i + 1]
        if b > a:
            _exact_rows(c, s, i, length - (b - a) + 1, out[a:b], lse[a:b])
    return out, lse
