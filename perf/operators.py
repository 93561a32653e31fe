"""The 8-bit serving operators, at the sizes they are used at.

Each case is one pass through the public entry points of
``paper_2311_14114_amd``, or through the same mathematics in elementary torch
operations.  The kinds:

  linear   a linear layer on 8-bit weights with one scale per output channel:
           its tokens quantized (one scale each), multiplied in integers and
           scaled into the output (``soniq_quantize_i8_gemm``)
  append   the keys and values of new tokens quantized into a paged cache
           (``soniq_kv_write``) and the rows just written read back
           (``soniq_kv_read``), as the chunk that follows sees them
  gather   cached sequences read back whole (``soniq_kv_read``), as a prompt
           on top of a cached prefix needs them
  attend   attention of new tokens over the paged cache
           (``soniq_kv_attention``): one token a sequence, a few in a row, or
           a tree of drafted tokens

A cache row is one position of one key/value head: ``head_dim`` codes of 8 or
4 bits in two's complement (4 bits: element 2i in the low half of byte i) and
one float32 scale, in pages of ``page`` rows per head:
codes ``[pages, heads, page, head_dim * bits / 8]``, scales
``[pages, heads, page]``.  Activations are N(0,1) with 1% of the channels 20
times larger, as in transformer encoders; weights are N(0, 0.02).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def _linear(name, M, N, K, *, dtype="bf16", bias=False, gap=0):
    """gap: columns between a token's last channel and the next token's first."""
    return dict(name=name, kind="linear", M=M, N=N, K=K, dtype=dtype, bias=bias, gap=gap)


def _append(name, B, lo, hi, heads, head_dim, bits, page, *, before=0, dtype="bf16"):
    """lo..hi new tokens for each of B sequences that hold up to `before` tokens."""
    return dict(name=name, kind="append", B=B, lo=lo, hi=hi, heads=heads, head_dim=head_dim, bits=bits,
                page=page, before=before, dtype=dtype)


def _gather(name, B, lo, hi, heads, head_dim, bits, page, *, dtype="bf16"):
    return dict(name=name, kind="gather", B=B, lo=lo, hi=hi, heads=heads, head_dim=head_dim, bits=bits,
                page=page, before=0, dtype=dtype)


def _attend(name, B, lo, hi, new, heads, group, head_dim, bits, page, *, tree=False, dtype="bf16"):
    """B sequences of lo..hi cached positions, the last `new` of them the new tokens'; `group` query heads a
    key/value head."""
    return dict(name=name, kind="attend", B=B, lo=lo, hi=hi, new=new, heads=heads, group=group,
                head_dim=head_dim, bits=bits, page=page, tree=tree, dtype=dtype)


def listed():
    return [
        # one token through a 4096-wide projection: what a decode step pays per layer
        _linear("linear_token", 1, 4096, 4096),
        # eight sequences with a short draft each, through the up projection of a 4096-wide decoder
        _linear("linear_drafts", 40, 11008, 4096),
        # a ragged prompt batch with sizes that no tile divides, a bias, and rows that start anywhere
        _linear("linear_odd", 301, 4099, 4091, dtype="fp16", bias=True, gap=5),
        # a prompt through the down projection
        _linear("linear_prompt", 4096, 4096, 11008),
        # compute-bound, the largest
        _linear("linear_square", 8192, 8192, 8192),
        # one new token for each of 32 sequences: the write that every decode step makes
        _append("append_tokens", 32, 1, 1, 8, 128, 8, 16, before=4000),
        # a batch of prompts written at once into a 4-bit cache
        _append("append_prompts", 5, 700, 4096, 8, 128, 4, 64, dtype="fp16"),
        # cached prefixes read back for a dense prompt pass
        _gather("gather_prefixes", 8, 1000, 16384, 8, 128, 8, 64),
        # a short prefix of an odd length from a small 4-bit cache, in float32
        _gather("gather_short", 1, 333, 333, 4, 64, 4, 16, dtype="fp32"),
        # one sequence, one token: the smallest attention call of a decode step
        _attend("attend_token", 1, 2049, 2049, 1, 8, 4, 128, 8, 16),
        # a full decode batch over long, ragged contexts: bound by the cache's bytes
        _attend("attend_batch", 32, 2000, 32768, 1, 8, 4, 128, 8, 64),
        # a tree of 24 drafted tokens for each of 8 sequences over a 4-bit cache
        _attend("attend_tree", 8, 3001, 8191, 24, 8, 4, 128, 4, 32, tree=True, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "append", "gather", "attend", "attend"])
    dtype = rng.choice(["bf16", "fp16"])
    heads, head_dim = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128, 128, 192, 256])
    bits, page = rng.choice([4, 8]), rng.choice([1, 8, 16, 16, 24, 32, 64, 128])
    row = heads * head_dim
    if kind == "linear":
        while True:
            M, N, K = _log(rng, 1, 8192), _log(rng, 64, 14336), _log(rng, 64, 14336)
            if rng.random() < 0.6:  # most models' widths; the rest as they fall
                N, K = -(-N // 128) * 128, -(-K // 128) * 128
            if 2 * M * N * K <= 5e11:
                return dict(kind=kind, M=M, N=N, K=K, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                            bias=rng.random() < 0.3, gap=rng.choice([0, 0, 0, 3, 64]))
    if kind in ("append", "gather"):
        while True:
            B, hi = _log(rng, 1, 64), _log(rng, 1, 16384)
            if B * hi * row <= 6e7:
                break
        lo = rng.randint(max(1, hi // 4), hi)
        if kind == "gather":
            return dict(kind=kind, B=B, lo=lo, hi=hi, heads=heads, head_dim=head_dim, bits=bits, page=page,
                        before=0, dtype=rng.choice(["bf16", "fp16", "fp32"]))
        return dict(kind=kind, B=B, lo=lo, hi=hi, heads=heads, head_dim=head_dim, bits=bits, page=page,
                    before=rng.choice([0, 100, 1000]), dtype=rng.choice(["bf16", "fp16", "fp32"]))
    new, tree = rng.choice([1, 1, 1, 2, 5, 16, 40, 64]), rng.random() < 0.5
    group = rng.choice([1, 4, 5, 8])
    while True:
        B, hi = _log(rng, 1, 64), _log(rng, max(16, new), 65536)
        if B * hi * row <= 3e8:
            break
    lo = rng.randint(max(new, hi // 8), hi)
    return dict(kind=kind, B=B, lo=lo, hi=hi, new=new, heads=heads, group=group, head_dim=head_dim, bits=bits,
                page=page, tree=tree and new > 1, dtype=dtype)


def _lengths(c):
    """The sequences' lengths (attend, gather) or their numbers of new tokens (append): spread over lo..hi, the
    longest one among them."""
    r = random.Random(c["B"] * 131 + c["hi"])
    return [c["hi"]] + [r.randint(c["lo"], c["hi"]) for _ in range(c["B"] - 1)]


def _befores(c):
    r = random.Random(c["B"] * 17 + c["before"])
    return [r.randint(0, c["before"]) for _ in range(c["B"])]


def work(c):
    if c["kind"] == "linear":
        M, N, K, e = c["M"], c["N"], c["K"], _SIZE[c["dtype"]]
        return {"bytes": M * K * e + N * K + 4 * N * (2 if c["bias"] else 1) + M * N * e, "flops": 2 * M * N * K}
    n = sum(_lengths(c))
    e, row = _SIZE[c["dtype"]], c["head_dim"] * c["bits"] // 8 + 4
    if c["kind"] == "append":  # rows in, codes and values out
        return {"bytes": 2 * n * c["heads"] * (2 * c["head_dim"] * e + row), "flops": 6 * n * c["heads"] * c["head_dim"]}
    if c["kind"] == "gather":
        return {"bytes": 2 * n * c["heads"] * (c["head_dim"] * e + row), "flops": 2 * n * c["heads"] * c["head_dim"]}
    rows = c["new"] * c["group"] * c["heads"]
    return {"bytes": 2 * n * c["heads"] * row + 2 * c["B"] * rows * c["head_dim"] * e,
            "flops": 4 * n * rows * c["head_dim"]}


def _pages(c, lengths, seed):
    """(pages, page table): every sequence's pages, scattered over the cache."""
    need = [-(-n // c["page"]) for n in lengths]
    total, width = sum(need) + 3, max(need)
    order = np.random.RandomState(seed % 2**31).permutation(total)
    table = np.zeros((c["B"], width), np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return total, torch.from_numpy(table).cuda()


def _prefix(counts):
    return torch.tensor([0, *np.cumsum(counts).tolist()], dtype=torch.int32, device="cuda")


def _cache(c, pages, g, filled):
    """Codes and scales of a cache: of standard normal rows, or empty."""
    shape = (pages, c["heads"], c["page"])
    width = c["head_dim"] * c["bits"] // 8
    s = {}
    for x in ("k", "v"):
        if not filled:
            s[x] = torch.zeros((*shape, width), dtype=torch.int8, device="cuda")
            s[x + "_scale"] = torch.zeros(shape, device="cuda")
            continue
        if c["bits"] == 8:
            codes = torch.empty((*shape, width), dtype=torch.float16, device="cuda").normal_(0, 36, generator=g)
            s[x] = codes.round_().clamp_(-127, 127).to(torch.int8)
        else:
            codes = torch.randint(-7, 8, (*shape, width, 2), dtype=torch.int8, device="cuda", generator=g)
            s[x] = (codes[..., 0] & 15) | (codes[..., 1] << 4)
        spread = torch.empty(shape, device="cuda").normal_(0, 0.2, generator=g).exp_()
        s[x + "_scale"] = spread.mul_(1 / 36 if c["bits"] == 8 else 1 / 4)
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _TYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        A = torch.randn((M, K + c["gap"]), device="cuda", generator=g)
        A[:, torch.rand(K + c["gap"], device="cuda", generator=g) < 0.01] *= 20
        s["A"] = A.to(dt)[:, :K]
        W = torch.randn((N, K), device="cuda", generator=g) * 0.02
        s["s_w"] = W.abs().amax(1) / 127
        s["W"] = (W / s["s_w"][:, None]).round_().clamp_(-127, 127).to(torch.int8)
        s["bias"] = torch.randn(N, device="cuda", generator=g) if c["bias"] else None
        return s
    lengths = _lengths(c)
    if c["kind"] == "append":
        before = _befores(c)
        pages, s["table"] = _pages(c, [a + n for a, n in zip(before, lengths)], seed)
        s["start"] = torch.tensor(before, dtype=torch.int32, device="cuda")
        s["cu"] = _prefix(lengths)
        s.update(_cache(c, pages, g, False))
        n = sum(lengths)
        # keys and values as a fused projection leaves them: side by side, per token
        kv = torch.randn((n, 2, c["heads"], c["head_dim"]), device="cuda", generator=g)
        kv *= torch.empty((1, 2, c["heads"], c["head_dim"]), device="cuda").normal_(0, 0.5, generator=g).exp_()
        kv = kv.to(dt)
        s["K"], s["V"] = kv[:, 0], kv[:, 1]
        s["tokens"] = n
        return s
    pages, s["table"] = _pages(c, lengths, seed)
    s.update(_cache(c, pages, g, True))
    if c["kind"] == "gather":
        s["start"] = torch.zeros(c["B"], dtype=torch.int32, device="cuda")
        s["cu"] = _prefix(lengths)
        s["tokens"] = sum(lengths)
        return s
    s["kv_len"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["cu"] = _prefix([c["new"]] * c["B"])
    s["max_kv"] = max(lengths)
    q = torch.randn((c["B"] * c["new"], c["heads"] * c["group"], c["head_dim"]), device="cuda", generator=g)
    s["q"] = (2 * q).to(dt)
    s["mask"] = None
    if c["tree"]:  # each drafted token sees itself and its ancestors; a token's parent is any earlier one
        r = random.Random(seed)
        words = []
        for _ in range(c["B"]):
            seen = []
            for i in range(c["new"]):
                p = r.randint(max(-1, i - 6), i - 1)
                seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            words += [w - (1 << 64) if w >= 1 << 63 else w for w in seen]
        s["mask"] = torch.tensor(words, dtype=torch.int64, device="cuda")[:, None]
    return s


# ---- the framework's calls ------------------------------------------------
def _own_cache(s):
    """The handle on the cache's tensors, made once, as a serving program does."""
    import paper_2311_14114_amd as sq
    if "handle" not in s:
        s["handle"] = sq.KVCache(s["k"], s["k_scale"], s["v"], s["v_scale"], bits=s["case"]["bits"])
    return sq, s["handle"]


def _run_own(s):
    c = s["case"]
    dt = _TYPES[c["dtype"]]
    if c["kind"] == "linear":
        import paper_2311_14114_amd as sq
        return sq.soniq_quantize_i8_gemm(s["A"], s["W"], s["s_w"], bias=s["bias"], dtype=dt)
    sq, cache = _own_cache(s)
    if c["kind"] == "append":
        sq.soniq_kv_write(cache, s["K"], s["V"], s["table"], s["cu"], s["start"])
        return sq.soniq_kv_read(cache, s["table"], s["cu"], s["start"], s["tokens"], dtype=dt)
    if c["kind"] == "gather":
        return sq.soniq_kv_read(cache, s["table"], s["cu"], s["start"], s["tokens"], dtype=dt)
    return sq.soniq_kv_attention(cache, s["q"], s["table"], s["cu"], s["kv_len"], mask=s["mask"],
                                 max_q=c["new"], max_kv=s["max_kv"])


# ---- the plain forms ------------------------------------------------------
def _quantize(x, top):
    """Codes (as float32) and scales of the rows of x: rint(x / s), s = max |x| / top; a row of zeros has
    scale 0 and codes 0."""
    x = x.float()
    s = x.abs().amax(-1, keepdim=True)
    s = s / torch.full_like(s, top)  # a division: by a number, torch multiplies with its reciprocal
    return torch.where(s > 0, torch.round(x / s), torch.zeros((), device=x.device)), s


def _rows(s, count):
    """The page, and the row inside it, of each new or cached position that cu and start name, in order."""
    c = s["case"]
    at = torch.arange(count, device="cuda")
    b = torch.searchsorted(s["cu"][1:].long(), at, right=True)
    pos = at - s["cu"].long()[b] + s["start"].long()[b]
    return s["table"].long()[b, pos // c["page"]], pos % c["page"]


def _unpack(codes, bits):
    if bits == 8:
        return codes.float()
    return torch.stack(((codes << 4) >> 4, codes >> 4), -1).flatten(-2).float()


def _values(s, x, page, row, dt):
    codes = _unpack(s[x][page, :, row], s["case"]["bits"])
    return (codes * s[x + "_scale"][page, :, row][..., None]).to(dt)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    dt = _TYPES[c["dtype"]]
    if c["kind"] == "linear":
        q, sa = _quantize(s["A"], 127.0)
        acc = (q.double() @ s["W"].double().t()).float()  # sums of integers past 2^24
        y = acc * sa * s["s_w"]
        return (y + s["bias"] if s["bias"] is not None else y).to(dt)
    if c["kind"] in ("append", "gather"):
        page, row = _rows(s, s["tokens"])
        if c["kind"] == "append":
            top = 127.0 if c["bits"] == 8 else 7.0
            for x, rows in (("k", s["K"]), ("v", s["V"])):
                q, sc = _quantize(rows, top)
                q = q.to(torch.int8)
                s[x][page, :, row] = q if c["bits"] == 8 else (q[..., 0::2] & 15) | (q[..., 1::2] << 4)
                s[x + "_scale"][page, :, row] = sc[..., 0]
        return _values(s, "k", page, row, dt), _values(s, "v", page, row, dt)
    # attend: the sequences padded to the longest one
    B, H, G, D, n, L = c["B"], c["heads"], c["group"], c["head_dim"], c["new"], s["max_kv"]
    pos = torch.arange(L, device="cuda")
    page, row = s["table"].long()[:, pos // c["page"]], (pos % c["page"])[None].expand(B, L)
    K = _values(s, "k", page, row, torch.float32).transpose(1, 2).reshape(B * H, L, D)
    V = _values(s, "v", page, row, torch.float32).transpose(1, 2).reshape(B * H, L, D)
    q = s["q"].float().view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B * H, n * G, D)
    S = torch.bmm(q, K.transpose(1, 2).contiguous()).view(B, H, n, G, L) / math.sqrt(D)
    new = pos[None] - (s["kv_len"].long()[:, None] - n)  # index among the new tokens, negative for older ones
    i = torch.arange(n, device="cuda")[None, :, None]
    if c["tree"]:
        seen = (s["mask"].view(B, n, 1) >> new[:, None].clamp(0, 63)) & 1 == 1
    else:
        seen = new[:, None] <= i
    seen = (new[:, None] < 0) | (seen & (new[:, None] < n))
    S = S.masked_fill(~seen[:, None, :, None], -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    O = torch.bmm(P.view(B * H, n * G, L), V)
    return O.view(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B * n, H * G, D).to(dt)


# ---- the definitions in 64 bits -------------------------------------------
def _exact_codes(x, top):
    """Scales are stored as float32, and a code is the integer nearest to the float32 quotient (even on ties)."""
    x = x.double()
    s = (x.abs().amax(-1, keepdim=True) / top).float().double()
    return torch.nan_to_num((x / s).float().double()).round(), s


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "linear":
        q, sa = _exact_codes(s["A"], 127.0)
        y = (q @ s["W"].double().t()) * (sa * s["s_w"].double()[None, :])
        return y if s["bias"] is None else y + s["bias"].double()
    if c["kind"] == "append":
        top = 127.0 if c["bits"] == 8 else 7.0
        out = []
        for x in ("K", "V"):
            q, sc = _exact_codes(s[x], top)
            out.append(q * sc)
        return tuple(out)
    lengths, outs = _lengths(c), {"k": [], "v": [], "o": []}
    for b, n in enumerate(lengths):
        t = s["table"][b, :-(-n // c["page"])].long()
        kv = []
        for x in ("k", "v"):
            byte = s[x][t].transpose(0, 1).reshape(c["heads"], -1, s[x].shape[-1])[:, :n].to(torch.int32)
            if c["bits"] == 4:
                lo, hi = byte & 15, (byte >> 4) & 15
                byte = torch.stack((lo - 16 * (lo > 7), hi - 16 * (hi > 7)), -1).reshape(c["heads"], n, -1)
            sc = s[x + "_scale"][t].transpose(0, 1).reshape(c["heads"], -1)[:, :n].double()
            kv.append(byte.double() * sc[..., None])
        if c["kind"] == "gather":
            outs["k"].append(kv[0].transpose(0, 1))
            outs["v"].append(kv[1].transpose(0, 1))
            continue
        m, G = c["new"], c["group"]
        q = s["q"][b * m:(b + 1) * m].double().view(m, c["heads"], G, -1)
        z = torch.matmul(q.permute(1, 0, 2, 3).reshape(c["heads"], m * G, -1), kv[0].transpose(1, 2).contiguous())
        z = z.view(c["heads"], m, G, n) / math.sqrt(c["head_dim"])
        hidden = torch.zeros((m, n), dtype=torch.bool)
        for i in range(m):
            for j in range(m):
                word = int(s["mask"][b * m + i, 0]) if c["tree"] else 0
                hidden[i, n - m + j] = not (word >> j) & 1 if c["tree"] else j > i
        z[hidden.cuda()[None, :, None].expand_as(z)] = -math.inf
        o = torch.matmul(torch.softmax(z, -1).view(c["heads"], m * G, n), kv[1])
        outs["o"].append(o.view(c["heads"], m, G, -1).permute(1, 0, 2, 3).reshape(m, c["heads"] * G, -1))
    if c["kind"] == "gather":
        return torch.cat(outs["k"]), torch.cat(outs["v"])
    return torch.cat(outs["o"])
