"""The serving operators of this library as cases that can be timed and compared: the product in 8-bit integers with a scale
for each token and each channel, and attention over a key/value cache held in 4-bit block floating point with the write
that fills it.

``run(state)`` makes either the library's calls (``own`` true) or the same operators in elementary torch operations.
``exact(case, seed)`` is the result from the definitions in 64 bits.

Kinds of work:
  int8     ``int8_gemm(x, w, bias)``: rows of activations quantised by the call, weights quantised ahead of time
  append   ``kv4_append`` then ``kv4_read``: new tokens' keys and values into the paged cache, and their values back
  attend   ``kv4_attention``: queries (one or several per sequence) against the paged cache

The cache. A page holds ``page`` tokens of every KV head; token t of a sequence lies in page ``table[t // page]``, row
``t % page``. A row of D values is D / 32 blocks of 32; a block is 32 mantissas of 4 bits and one exponent s (int8):
value = (nibble - 8) * 2^s. Every 32-bit word holds eight consecutive values, value 2 i in nibble i and value 2 i + 1 in
nibble i + 4. Arrays: mantissas uint8 [pages][heads][page][D / 2], exponents int8 [pages][heads][page][D / 32].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# ----------------------------------------------------------------------------- cases


def listed():
    return [
        # a projection for one token of one sequence: latency and reading the weights
        dict(name="int8_1_row", kind="int8", M=1, N=4096, K=4096, dtype="bf16", bias=False),
        # a batch of sixteen decoding sequences, the shape of the benchmark's serving product, FP32 activations
        dict(name="int8_16_rows", kind="int8", M=16, N=4096, K=4096, dtype="f32", bias=True),
        # a layer whose extents fit no tile, vector or row pitch
        dict(name="int8_ragged", kind="int8", M=1111, N=777, K=3001, dtype="f16", bias=True),
        # the feed-forward projection of the transformer configuration: 4096 tokens, 1024 -> 4096
        dict(name="int8_ffn", kind="int8", M=4096, N=4096, K=1024, dtype="f32", bias=True),
        # the prefill of a large layer: bound by the tensor cores
        dict(name="int8_8192", kind="int8", M=8192, N=8192, K=8192, dtype="bf16", bias=False),
        # one decode step of 64 sequences: 64 tokens into 64 different pages
        dict(name="append_step", kind="append", B=64, n=1, lo=1, hi=4096, heads=8, D=128, page=64, dtype="bf16"),
        # prompts of 8 sequences, of different lengths, written at once
        dict(name="append_prompts", kind="append", B=8, n=1024, lo=1024, hi=4096, heads=8, D=128, page=16, dtype="f32"),
        # a few short conversations in a small network: latency
        dict(name="attend_small", kind="attend", B=4, n=1, lo=1, hi=300, heads=4, group=1, D=64, page=16, window=0, dtype="f32"),
        # a serving batch of 64 sequences of up to 8192 tokens, grouped heads: bound by reading the cache
        dict(name="attend_batch", kind="attend", B=64, n=1, lo=500, hi=8192, heads=8, group=4, D=128, page=64, window=0, dtype="bf16"),
        # one sequence with a very long context: too few heads to fill the chip unless the keys are split
        dict(name="attend_long", kind="attend", B=1, n=1, lo=131072, hi=131072, heads=8, group=8, D=128, page=128, window=0, dtype="f16"),
        # five drafted tokens a sequence, three query heads to a KV head, odd lengths, a sliding window
        dict(name="attend_drafts", kind="attend", B=7, n=5, lo=100, hi=5001, heads=2, group=3, D=96, page=32, window=1000, dtype="f32"),
        # prompts of 2048 tokens behind cached prefixes: bound by arithmetic
        dict(name="attend_prompts", kind="attend", B=2, n=2048, lo=2048, hi=4096, heads=8, group=4, D=128, page=64, window=0, dtype="bf16"),
    ]


_MOST_PRODUCT = 8192 ** 3
_MOST_CACHE = 64 * 8 * 128 * 4352        # values of a cache that one call reads: the listed batch's
_MOST_SCORES = 64 * 2048 * 2500          # scores of a call with many queries


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]: any value, or one rounded to a multiple of 8 or 64."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice((1, 1, 8, 64))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(("int8", "int8", "append", "attend", "attend", "attend"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if kind == "int8":
        while True:
            M, N, K = _log(rng, 1, 8192), _log(rng, 16, 16384), _log(rng, 16, 16384)
            if M * N * K <= _MOST_PRODUCT // 2:
                return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, bias=rng.choice((False, True)))
    D, page = rng.choice((64, 96, 128, 128, 256)), rng.choice((16, 32, 64, 64, 128, 256))
    heads = rng.choice((1, 2, 4, 8, 8, 16))
    if kind == "append":
        while True:
            B, n = _log(rng, 1, 256), rng.choice((1, 1, _log(rng, 2, 2048)))
            if B * n * heads * D <= 1 << 23:
                lo = n + _log(rng, 1, 1024) - 1
                return dict(kind=kind, B=B, n=n, lo=lo, hi=lo + _log(rng, 1, 2048), heads=heads, D=D, page=page, dtype=dtype)
    group = rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 12))
    while True:
        B, n = _log(rng, 1, 128), rng.choice((1, 1, 1, rng.randint(2, 9), _log(rng, 10, 1024)))
        lo = _log(rng, 1, 16384)
        hi = min(131072, lo * rng.choice((1, 1, 2, 4)))
        if n > 1:
            lo, hi = max(lo, n), max(hi, n)
        if B * heads * D * (lo + hi) <= _MOST_CACHE and (n == 1 or B * n * heads * group * (lo + hi) <= _MOST_SCORES):
            return dict(kind=kind, B=B, n=n, lo=lo, hi=hi, heads=heads, group=group, D=D, page=page,
                        window=rng.choice((0, 0, 0, _log(rng, 16, 4096))), dtype=dtype)


# ----------------------------------------------------------------------------- inputs


def _lengths(case):
    """Tokens of each sequence after the call, its own included: spread evenly over [lo, hi], the longest in the middle."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    if B == 1:
        return [hi]
    return [lo + (hi - lo) * ((i * 2 if 2 * i < B else 2 * (B - 1 - i) + 1)) // (B - 1) for i in range(B)]


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _inputs(case, seed):
    """What both sides and the exact result start from: plain tensors on the GPU, and the sequences' lengths on the host."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = _DTYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] == "int8":
        M, N, K = case["M"], case["N"], case["K"]
        x = _normal(gen, M, K)
        x *= torch.exp(0.5 * _normal(gen, M, 1))                   # tokens of different size
        x *= 1 + 19 * (torch.rand(1, K, generator=gen, device="cuda") < 0.004)       # a few channels with large values, as activations have them
        s["x"] = x.to(t)
        w = _normal(gen, N, K).mul_((2.0 / K) ** 0.5)
        # the scale of a channel and its integers, as the weights are laid out once: rows padded to 16 bytes with zeros
        scale = (w.abs().amax(1).double() / 127).float()
        q = torch.round(w.double() / scale.double()[:, None]).to(torch.int8)
        pitch = (K + 15) // 16 * 16
        s["wq"] = torch.zeros(N, pitch, dtype=torch.int8, device="cuda")
        s["wq"][:, :K] = q
        s["ws"] = scale
        s["bias"] = _normal(gen, N) if case["bias"] else None
        return s
    B, n, H, D, page = (case[k] for k in ("B", "n", "heads", "D", "page"))
    lengths = _lengths(case)
    per = [-(-v // page) for v in lengths]
    pages = sum(per)
    order = torch.randperm(pages, generator=gen, device="cuda")    # the pages of a sequence lie anywhere
    table = torch.full((B, max(per)), -1, dtype=torch.int32, device="cuda")        # -1: behind the sequence's last page
    at = 0
    for b, c in enumerate(per):
        table[b, :c] = order[at:at + c]
        at += c
    s.update(lengths_host=lengths, table=table, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), pages=pages)
    if case["kind"] == "append":
        # views of one fused projection's output: rows further apart than they are long
        kv = _normal(gen, B * n, 2 * H, D)
        kv *= torch.exp(_normal(gen, 1, 2 * H, D))                 # channels of different size
        kv = kv.to(t)
        s["k"], s["v"] = kv[:, :H], kv[:, H:]
        s["arrays"] = _empty_cache(pages, H, page, D)
        return s
    G = case["group"]
    spread = torch.exp(0.5 * _normal(gen, 1, H, 1, D))
    s["arrays"] = _pack(_normal(gen, pages, H, page, D).mul_(spread)) + _pack(_normal(gen, pages, H, page, D))
    q = _normal(gen, B * n, H * G, D)
    q[..., : D // 2] *= 2.0
    s["q"] = q.to(t)
    s["scale"] = D ** -0.5
    return s


def _empty_cache(pages, H, page, D):
    return tuple(torch.zeros(pages, H, page, w, dtype=t, device="cuda") for w, t in
                 ((D // 2, torch.uint8), (D // 32, torch.int8)) * 2)


def _quantise(x):
    """Mantissas (float32 whole numbers) and exponents of blocks of 32 along the last axis, nearest-even."""
    x = x.float().unflatten(-1, (-1, 32))
    _, e = torch.frexp(x.abs().amax(-1))                           # amax = f * 2^e with f in [0.5, 1)
    s = torch.where(x.abs().amax(-1) > 0, e - 3, torch.full_like(e, -63)).clamp(-63, 120)
    q = torch.round(torch.ldexp(x, -s[..., None])).clamp_(-7, 7)
    return q, s


def _pack(x):
    """Values [..][D] to the cache's arrays: mantissas [..][D / 2], exponents [..][D / 32]."""
    q, s = _quantise(x)
    n = (q + 8).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 4, 2))              # word, pair, member: nibble pair + 4 * member
    n = n.transpose(-1, -2).flatten(-2).unflatten(-1, (4, 2))                      # byte, half
    return (n[..., 0] | (n[..., 1] << 4)).flatten(-2), s.to(torch.int8)


def _unpack(m, s):
    """The values (float32) of mantissa and exponent arrays."""
    n = torch.stack((m & 15, m >> 4), -1).unflatten(-2, (-1, 4)).flatten(-2)       # word, nibble
    n = n.unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-3)                      # the values in order
    return torch.ldexp((n.float() - 8).unflatten(-1, (-1, 32)), s.int()[..., None]).flatten(-2)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_1804_01526_b200 import binding as hb

        s["hb"] = hb
        if s["kind"] == "int8":
            s["w"] = hb.Int8Rows(s["wq"], s["ws"], s["K"])
        else:
            s["cache"] = hb.Kv4Cache(*s["arrays"])
    return s


# ----------------------------------------------------------------------------- one pass


def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


def _own_int8(s):
    return s["hb"].int8_gemm(s["x"], s["w"], bias=s["bias"])


def _own_append(s):
    s["hb"].kv4_append(s["cache"], s["k"], s["v"], s["table"], s["lengths"])
    return s["hb"].kv4_read(s["cache"], s["n"], s["table"], s["lengths"])


def _own_attend(s):
    return s["hb"].kv4_attention(s["q"], s["cache"], s["table"], s["lengths"], scale=s["scale"], window=s["window"])


def _plain_int8(s):
    x = s["x"]
    scale = (x.abs().amax(1).double() / 127).float()
    # a quotient next to a half is decided in 64 bits
    q = torch.round(x.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double()[:, None]).float()
    y = q @ s["wq"][:, :s["K"]].float().t()
    y = y * scale[:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(x.dtype)


def _plain_append(s):
    km, ke, vm, ve = s["arrays"]
    p = (s["lengths"][:, None] - s["n"] + torch.arange(s["n"], device="cuda")).long()        # positions of the new tokens
    pages, rows = s["table"].gather(1, p // s["page"]).flatten().long(), (p % s["page"]).flatten()
    outs = []
    for x, m, e in ((s["k"], km, ke), (s["v"], vm, ve)):
        m[pages, :, rows], e[pages, :, rows] = _pack(x)
        outs.append(_unpack(m[pages, :, rows], e[pages, :, rows]))
    return tuple(outs)


def _plain_attend(s):
    n, H, G, D, page, window = (s[k] for k in ("n", "heads", "group", "D", "page", "window"))
    km, ke, vm, ve = s["arrays"]
    out = torch.empty_like(s["q"])
    for b, L in enumerate(s["lengths_host"]):
        first = max(0, L - n - window + 1) // page * page if window else 0         # no key before it is seen
        ids = s["table"][b, first // page:-(-L // page)].long()
        k = _unpack(km[ids], ke[ids]).transpose(0, 1).flatten(1, 2)[:, :L - first]           # [H][keys][D]
        v = _unpack(vm[ids], ve[ids]).transpose(0, 1).flatten(1, 2)[:, :L - first]
        q = s["q"][b * n:(b + 1) * n].float().unflatten(1, (H, G)).permute(1, 2, 0, 3).flatten(1, 2)      # [H][G * n][D]
        x = (q @ k.transpose(1, 2)).mul_(s["scale"])
        j = torch.arange(first, L, device="cuda")
        i = torch.arange(L - n, L, device="cuda")[:, None]
        hidden = j > i
        if window:
            hidden |= j <= i - window
        x = x.unflatten(1, (G, n)).masked_fill_(hidden, -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        total = x.sum(-1, keepdim=True)
        o = (x.flatten(1, 2) @ v).unflatten(1, (G, n)) / total
        out[b * n:(b + 1) * n] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
    return out


_OWN = {"int8": _own_int8, "append": _own_append, "attend": _own_attend}
_PLAIN = {"int8": _plain_int8, "append": _plain_append, "attend": _plain_attend}


# ----------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "int8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": size * (M * K + M * N) + N * K + 4 * N * (2 if case["bias"] else 1), "flops": 2 * M * N * K}
    B, n, H, D = (case[k] for k in ("B", "n", "heads", "D"))
    row = D // 2 + D // 32                                         # bytes of a token's keys (or values) of one head
    if case["kind"] == "append":
        return {"bytes": 2 * B * n * H * (size * D + row + 4 * D), "flops": 0}
    window, lengths = case["window"], _lengths(case)
    keys = sum(L - max(0, L - n - window + 1) if window else L for L in lengths)
    seen = sum(min(i + 1, window) if window else i + 1 for L in lengths for i in range(L - n, L))
    return {"bytes": 2 * size * B * n * H * case["group"] * D + 2 * keys * H * row, "flops": 4 * D * H * case["group"] * seen}


# ----------------------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "int8":
        return _exact_int8(s)
    if case["kind"] == "append":
        return tuple(_exact_values(s[x]) for x in ("k", "v"))
    return _exact_attend(s)


def _exact_int8(s):
    x, K = s["x"].double(), s["K"]
    top = x.abs().max(dim=1).values
    scale = (top / 127.0).to(torch.float32).to(torch.float64)      # the scale is an FP32 number
    q = (x / scale.clamp_min(1e-300)[:, None]).round()             # half to even
    y = torch.matmul(q, s["wq"].double()[:, :K].T)                 # whole numbers below 2^53
    y = torch.einsum("mn,m,n->mn", y, scale, s["ws"].double())
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_values(x):
    x = x.double().cpu().numpy()
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(b).max(axis=-1, keepdims=True)
    e = np.frexp(top)[1]                                           # floor(log2 top) + 1
    s = np.where(top > 0, np.clip(e - 3, -63, 120), -63)
    q = np.clip(np.rint(b * np.exp2(-s.astype(np.float64))), -7, 7)
    return (q * np.exp2(s.astype(np.float64))).reshape(x.shape)


def _exact_attend(s):
    n, H, G, D, page = (s[k] for k in ("n", "heads", "group", "D", "page"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    km, ke, vm, ve = s["arrays"]
    value = torch.arange(8, device="cuda")
    place = 4 * (value // 2 + 4 * (value % 2))                     # bit at which each of a word's eight values starts

    def values(m, e, h, pages, rows):
        words = m[pages, h, rows].contiguous().view(torch.int32).long()
        mant = ((words[..., None] >> place) & 15) - 8
        two = torch.pow(2.0, e[pages, h, rows].double())
        return (mant.reshape(len(rows), D // 32, 32).double() * two[..., None]).reshape(len(rows), D)

    for b, L in enumerate(s["lengths_host"]):
        pos = torch.arange(L, device="cuda")
        pages, rows = s["table"][b].long()[pos // page], pos % page
        query = torch.arange(L - n, L, device="cuda")
        seen = pos[None, :] <= query[:, None]
        if s["window"]:
            seen &= query[:, None] - pos[None, :] < s["window"]
        for h in range(H):
            k, v = values(km, ke, h, pages, rows), values(vm, ve, h, pages, rows)
            for g in range(G):
                x = s["q"][b * n:(b + 1) * n, h * G + g].double() @ k.T * s["scale"]
                x = torch.where(seen, x, torch.full_like(x, -torch.inf))
                p = torch.exp(x - torch.logsumexp(x, dim=1, keepdim=True))
                out[b * n:(b + 1) * n, h * G + g] = p @ v
    return out
