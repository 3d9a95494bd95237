"""The paged key/value cache and the attention over it: what they cost a user, and what they compute in plain form.

Shapes are those of the attention block around workloads.CFG5_LINEARS (32 query heads and 8 key/value heads of 128) and
generic ones: heads of 64, every query head with keys of its own, few key/value heads for many query heads.

Paths ("path" of a case):

  append   sr_rope_kv_append of T new tokens, then sr_kv_gather of the rows they went to (the keys and values as the cache
           holds them, which the attention of a prompt goes on with)
  decode   sr_attn_decode: one new token of each sequence over its pages
  prefill  sr_attn_prefill: packed prompts, causal; with "prefix", the keys of earlier chunks in front

"kind" is what the cache holds: "i4" (asymmetric 4 bits, a scale and a zero per token and head) or "f16".
"""
from __future__ import annotations

import math
import random

import torch

own = False

CLIP = 0.95


def listed():
    return [
        # the new token of one sequence, keys turned by the Hadamard transform: latency
        dict(name="append_1_i4", path="append", T=1, H=32, KV=8, d=128, page=16, kind="i4", hadamard=True, pairs=False),
        # a decode step's tokens, one of each of 61 sequences, small heads, 16-bit cache, angles in pairs
        dict(name="append_61_f16", path="append", T=61, H=16, KV=2, d=64, page=32, kind="f16", hadamard=False, pairs=True),
        # a prompt of ordinary, odd length
        dict(name="append_2047_i4", path="append", T=2047, H=32, KV=8, d=128, page=64, kind="i4", hadamard=True, pairs=False),
        # packed long prompts: the largest append
        dict(name="append_16384_i4", path="append", T=16384, H=32, KV=8, d=128, page=64, kind="i4", hadamard=False, pairs=False),
        # one sequence, just begun: latency
        dict(name="decode_1_130_i4", path="decode", B=1, L=130, H=32, KV=8, d=128, page=16, kind="i4", ragged=0),
        # one long document: only the split over its length fills the chip
        dict(name="decode_1_65000_i4", path="decode", B=1, L=65000, H=32, KV=8, d=128, page=64, kind="i4", ragged=0),
        # a busy server: 64 sequences of every length up to 8192
        dict(name="decode_64_ragged_i4", path="decode", B=64, L=8192, H=32, KV=8, d=128, page=64, kind="i4", ragged=7),
        # every query head with keys of its own, small heads, 16-bit cache
        dict(name="decode_24_mha_f16", path="decode", B=24, L=2000, H=32, KV=32, d=64, page=32, kind="f16", ragged=5),
        # a short prompt
        dict(name="prefill_113", path="prefill", N=1, T=113, H=32, KV=8, d=128, ragged=0, prefix=0),
        # a batch of nine prompts of different lengths
        dict(name="prefill_packed_2500", path="prefill", N=9, T=2500, H=32, KV=8, d=128, ragged=3, prefix=0),
        # chunks of four long prompts behind what is cached of them, heads of 64
        dict(name="prefill_chunks_d64", path="prefill", N=4, T=1030, H=16, KV=2, d=64, ragged=2, prefix=1500),
        # one long prompt
        dict(name="prefill_8192", path="prefill", N=1, T=8192, H=32, KV=8, d=128, ragged=0, prefix=0),
    ]


HEADS = ((32, 8), (32, 8), (32, 32), (16, 2), (8, 1), (20, 4), (32, 1), (6, 6))


def draw(rng):
    path = rng.choice(["append", "decode", "prefill"])
    H, KV = rng.choice(HEADS)
    d = rng.choice([64, 128, 128])

    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    c = dict(path=path, H=H, KV=KV, d=d)
    if path == "append":
        # 16-bit rows are wider than the listed ones, and so are tokens of more heads
        c.update(T=spread(1, 12000 * 48 // max(48, H + 2 * KV)), page=rng.choice([16, 32, 64, 128]),
                 kind=rng.choice(["i4", "i4", "f16"]), hadamard=rng.random() < 0.5, pairs=rng.random() < 0.25)
    elif path == "decode":
        kind = rng.choice(["i4", "i4", "f16"])
        B = spread(1, 64)
        # rows of the cache and products at most those of the largest listed case; 16 bits are 3.6 times the bytes
        rows = 64 * 8192 * 8 // (2 if kind == "i4" else 8)
        c.update(B=B, L=spread(1, min(65000, rows // (KV * B), 64 * 8192 * 16 // (H * B))), page=rng.choice([16, 32, 64, 256]), kind=kind, ragged=rng.randrange(1 << 16))
    else:
        N = spread(1, 12)
        c.update(N=N, T=spread(12, 6000), ragged=rng.randrange(1, 1 << 16), prefix=rng.choice([0, 0, spread(1, 2400 // N)]))
    return c


# ---- lengths ---------------------------------------------------------------------------------------------------------

def cut(total, parts, rng):
    """`total` cut into `parts` lengths of one or more at random places."""
    at = sorted(rng.sample(range(1, total), parts - 1)) if parts > 1 else []
    return [b - a for a, b in zip([0] + at, at + [total])]


def decode_lens(c):
    """Every length from nothing (a padding row of the batch) to L, the longest always there."""
    if not c["ragged"]:
        return [c["L"]] * c["B"]
    rng = random.Random(c["ragged"])
    return [c["L"]] + [rng.randint(0, c["L"]) for _ in range(c["B"] - 1)]


def prefill_lens(c):
    """(query lengths, key lengths) of the packed sequences."""
    rng = random.Random(c["ragged"])
    q = cut(c["T"], c["N"], rng)
    return q, [n + (rng.randint(0, c["prefix"]) if c["prefix"] else 0) for n in q]


def row_bytes(c):
    """Bytes of one token and head in the cache."""
    return c["d"] // 2 + 8 if c["kind"] == "i4" else 2 * c["d"]


def work(c):
    H, KV, d = c["H"], c["KV"], c["d"]
    if c["path"] == "append":
        T = c["T"]
        read = T * ((H + 2 * KV) * d * 2 + d * 4 + 12)
        written = T * (H * d * 2 + 2 * KV * (row_bytes(c) + 2 * d))
        return {"bytes": read + written, "flops": T * (H + KV) * d * (3 + (math.log2(d) if c["hadamard"] else 0))}
    if c["path"] == "decode":
        tokens = sum(decode_lens(c))
        return {"bytes": tokens * 2 * KV * row_bytes(c) + c["B"] * H * d * 4, "flops": 4 * tokens * H * d}
    q, k = prefill_lens(c)
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q, k))
    return {"bytes": 2 * d * (2 * H * sum(q) + 2 * KV * sum(k)), "flops": 4 * pairs * H * d}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def quantised(x):
    """Asymmetric 4-bit codes of the last axis in 32 bits: (codes, scale, zero), the latter with that axis of size 1."""
    hi, lo = CLIP * x.amax(-1, keepdim=True), CLIP * x.amin(-1, keepdim=True)
    scale = torch.where(hi == lo, torch.ones_like(hi), (hi - lo) / 15)
    zero = -torch.round(lo / scale)
    return torch.clamp(torch.round(x / scale) + zero, 0, 15), scale, zero


def packed(codes):
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpacked(q):
    return torch.stack((q & 15, q >> 4), -1).flatten(-2)


def filled(shape, kind, offset, g):
    """One side of a cache whose pages hold normal values around an offset per channel: (rows, params)."""
    x = (torch.randn(shape, generator=g, device="cuda") + offset).half()
    if kind == "f16":
        return x, None
    codes, scale, zero = quantised(x.float())
    return packed(codes), torch.cat((scale, zero), -1)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H, KV, d = c["H"], c["KV"], c["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def shuffled(n):
        return torch.randperm(n, generator=g, device="cuda")

    k_offset, v_offset = 0.5 * normal(KV, 1, d), 0.1 * normal(KV, 1, d)
    if c["path"] == "append":
        T, page = c["T"], c["page"]
        # what the fused projection leaves: queries, keys and values of a token side by side
        x = normal(T, (H + 2 * KV) * d)
        x[:, H * d:(H + KV) * d] += k_offset.view(1, -1)
        x[:, (H + KV) * d:] += v_offset.view(1, -1)
        x = x.half()
        pages = -(-T // page) + 3
        cache = (filled((pages, KV, page, d), c["kind"], k_offset, g), filled((pages, KV, page, d), c["kind"], v_offset, g))
        at = torch.arange(T, device="cuda")
        slots = shuffled(pages)[at // page] * page + at % page
        # positions of one run of tokens that begins anywhere in a long context
        first = torch.randint(0, 1 << 15, (1,), generator=g, device="cuda")
        positions = (first + at).int()
        angle = torch.arange((1 << 15) + 16384, device="cuda", dtype=torch.float64)[:, None]
        angle = angle * 500000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        table = torch.cat((angle.cos(), angle.sin()), -1).float()
        return dict(c=c, q=x[:, :H * d], k=x[:, H * d:(H + KV) * d], v=x[:, (H + KV) * d:], positions=positions, slots=slots, table=table,
                    cache=(cache[0][0], cache[1][0], cache[0][1], cache[1][1]))
    if c["path"] == "decode":
        B, page, lens = c["B"], c["page"], decode_lens(c)
        width = max(1, -(-max(lens) // page))
        used = [-(-n // page) for n in lens]
        pages = sum(used) + 1
        order, table, at = shuffled(pages).int(), torch.full((B, width), -1, dtype=torch.int32, device="cuda"), 0
        for b, n in enumerate(used):
            table[b, :n] = order[at:at + n]
            at += n
        cache = (filled((pages, KV, page, d), c["kind"], k_offset, g), filled((pages, KV, page, d), c["kind"], v_offset, g))
        return dict(c=c, q=(1.5 * normal(B, H * d)).half(), table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    cache=(cache[0][0], cache[1][0], cache[0][1], cache[1][1]))
    ql, kl = prefill_lens(c)
    ends = [torch.tensor([0] + n, dtype=torch.int32, device="cuda").cumsum(0).int() for n in (ql, kl)]
    k = normal(sum(kl), KV, d) + k_offset.view(1, KV, d)
    v = normal(sum(kl), KV, d) + v_offset.view(1, KV, d)
    return dict(c=c, q=(1.5 * normal(sum(ql), H * d)).half(), k=k.half().flatten(1), v=v.half().flatten(1), cu_q=ends[0], cu_k=ends[1])


# ---- plain forms -----------------------------------------------------------------------------------------------------

def rotated(x, s, heads):
    """x [T, heads * d] turned by the angles of its positions and, where asked, by the Hadamard matrix inside each head."""
    c = s["c"]
    d, T = c["d"], x.shape[0]
    cos, sin = s["table"][s["positions"].long()].view(T, 1, 2, d // 2).unbind(2)
    x = x.float().view(T, heads, d)
    if c["pairs"]:
        a, b = x[..., 0::2], x[..., 1::2]
    else:
        a, b = x[..., :d // 2], x[..., d // 2:]
    y = (a * cos - b * sin, b * cos + a * sin)
    x = torch.stack(y, -1).flatten(-2) if c["pairs"] else torch.cat(y, -1)
    if c["hadamard"]:
        h = 1
        while h < d:
            a, b = x.view(T, heads, -1, 2, h).unbind(3)
            x, h = torch.stack((a + b, a - b), 3).view(T, heads, d), 2 * h
        x = x * (1 / math.sqrt(d))
    return x.half()


def plain_append(s):
    c = s["c"]
    H, KV, d, page = c["H"], c["KV"], c["d"], c["page"]
    k, v = rotated(s["k"], s, KV), s["v"].view(-1, KV, d)
    at, off = s["slots"] // page, s["slots"] % page
    K, V, Kp, Vp = s["cache"]
    if c["kind"] == "f16":
        K[at, :, off], V[at, :, off] = k, v
        return rotated(s["q"], s, H).flatten(1), K[at, :, off].flatten(1), V[at, :, off].flatten(1)
    (kc, ks, kz), (vc, vs, vz) = quantised(k.float()), quantised(v.float())
    K[at, :, off], V[at, :, off] = packed(kc), packed(vc)
    Kp[at, :, off], Vp[at, :, off] = torch.cat((ks, kz), -1), torch.cat((vs, vz), -1)
    return rotated(s["q"], s, H).flatten(1), of_rows(K[at, :, off], Kp[at, :, off]).half().flatten(1), of_rows(V[at, :, off], Vp[at, :, off]).half().flatten(1)


def of_rows(rows, params):
    """The values that rows of a cache stand for, in 32 bits."""
    return rows.float() if params is None else (unpacked(rows).float() - params[..., 1:]) * params[..., :1]


def softmax_product(scores, V):
    """Rows of scores (minus infinity where masked) times V; a row without a score gives zeros."""
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return (p @ V) / torch.where(total == 0, torch.ones_like(total), total)


def plain_decode(s):
    c = s["c"]
    H, KV, d, B = c["H"], c["KV"], c["d"], c["B"]
    at = s["table"].long().clamp(min=0)
    K, V, Kp, Vp = s["cache"]
    K = of_rows(K[at], None if Kp is None else Kp[at]).transpose(1, 2).reshape(B, KV, -1, d)
    V = of_rows(V[at], None if Vp is None else Vp[at]).transpose(1, 2).reshape(B, KV, -1, d)
    scores = s["q"].float().view(B, KV, H // KV, d) @ K.transpose(2, 3).contiguous() * (1 / math.sqrt(d))
    gone = torch.arange(K.shape[2], device="cuda") >= s["lens"].view(B, 1, 1, 1)
    return softmax_product(scores.masked_fill(gone, -math.inf), V).reshape(B, H * d).half()


def plain_prefill(s):
    c = s["c"]
    H, KV, d = c["H"], c["KV"], c["d"]
    cq, ck = s["cu_q"], s["cu_k"]
    i, j = torch.arange(s["q"].shape[0], device="cuda"), torch.arange(s["k"].shape[0], device="cuda")
    sq, sk = torch.searchsorted(cq[1:], i.int(), right=True), torch.searchsorted(ck[1:], j.int(), right=True)
    # counted from the ends of their sequences, which lie on each other
    behind_q, behind_k = cq[sq + 1] - i, ck[sk + 1] - j
    gone = (sq[:, None] != sk[None, :]) | (behind_k[None, :] < behind_q[:, None])
    q = s["q"].float().view(-1, KV, H // KV, d).permute(1, 2, 0, 3).flatten(1, 2)
    K, V = (s[n].float().view(-1, KV, d).transpose(0, 1).contiguous() for n in "kv")
    scores = (q @ K.transpose(1, 2).contiguous()).view(KV, H // KV, len(i), len(j)).mul_(1 / math.sqrt(d)).masked_fill_(gone, -math.inf)
    out = softmax_product(scores.flatten(1, 2), V).view(KV, H // KV, len(i), d)
    return out.permute(2, 0, 1, 3).reshape(len(i), H * d).half()


def own_append(s):
    import paper_2506_05413_amd as sr
    c = s["c"]
    q = sr.sr_rope_kv_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["table"], s["cache"], hadamard=c["hadamard"], pairs=c["pairs"], clip=CLIP)
    return (q, *sr.sr_kv_gather(s["slots"], s["cache"]))


def own_decode(s):
    import paper_2506_05413_amd as sr
    return sr.sr_attn_decode(s["q"], s["cache"], s["table"], s["lens"])


def own_prefill(s):
    import paper_2506_05413_amd as sr
    return sr.sr_attn_prefill(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["c"]["d"])


def run(s):
    path = s["c"]["path"]
    if own:
        return own_append(s) if path == "append" else own_decode(s) if path == "decode" else own_prefill(s)
    return plain_append(s) if path == "append" else plain_decode(s) if path == "decode" else plain_prefill(s)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def exact_attention(q, k, v, shift):
    """One sequence, one key/value head: q [n, d] of 64 bits, row i sees the keys j <= i + shift."""
    n, m = q.shape[0], k.shape[0]
    w = q @ k.T.contiguous() / math.sqrt(q.shape[1])
    w = w.masked_fill(torch.ones(n, m, dtype=torch.bool, device=q.device).triu(shift + 1), -math.inf)
    return torch.softmax(w, -1) @ v if m else torch.zeros_like(q)


def exact_values(rows, params):
    if params is None:
        return rows.double()
    out = torch.empty((*rows.shape[:-1], 2 * rows.shape[-1]), dtype=torch.float64, device=rows.device)
    out[..., 0::2], out[..., 1::2] = (rows % 16).double(), (rows // 16).double()
    return (out - params[..., 1:].double()) * params[..., :1].double()


def exact_rotation(x, s, heads):
    c = s["c"]
    d = c["d"]
    rows = s["table"].double()[s["positions"].long()]
    first = torch.arange(0, d, 2) if c["pairs"] else torch.arange(d // 2)
    second = first + (1 if c["pairs"] else d // 2)
    turn = torch.zeros(len(rows), d, d, dtype=torch.float64, device="cuda")
    i = torch.arange(d // 2)
    turn[:, first, first], turn[:, second, second] = rows[:, i], rows[:, i]
    turn[:, second, first], turn[:, first, second] = -rows[:, d // 2 + i], rows[:, d // 2 + i]
    if c["hadamard"]:
        bits = torch.tensor([[bin(a & b).count("1") & 1 for b in range(d)] for a in range(d)], device="cuda")
        turn = turn @ ((1.0 - 2.0 * bits.double()) / math.sqrt(d))
    return (x.double().view(-1, heads, d) @ turn).flatten(1)


def exact(c, seed):
    s = prepare(c, seed)
    H, KV, d = c["H"], c["KV"], c["d"]
    G = H // KV
    if c["path"] == "append":
        out = [[], [], []]
        for a in range(0, c["T"], 1024):
            part = dict(s, positions=s["positions"][a:a + 1024])
            out[0].append(exact_rotation(s["q"][a:a + 1024], part, H))
            for n, x in ((1, exact_rotation(s["k"][a:a + 1024], part, KV)), (2, s["v"][a:a + 1024].double())):
                x = x.half().double().view(-1, KV, d)  # keys and values reach the cache in 16 bits
                if c["kind"] == "i4":
                    clip = torch.tensor(CLIP).double().item()
                    hi, lo = clip * x.max(-1, keepdim=True).values, clip * x.min(-1, keepdim=True).values
                    step = (hi - lo) / 15
                    step[step == 0] = 1
                    shift = torch.round(lo / step)
                    x = ((torch.round(x / step) - shift).clamp(0, 15) + shift) * step
                out[n].append(x.flatten(1))
        return tuple(torch.cat(x) for x in out)
    if c["path"] == "decode":
        K, V, Kp, Vp = s["cache"]
        out = torch.zeros(c["B"], H, d, dtype=torch.float64, device="cuda")
        for b, n in enumerate(decode_lens(c)):
            at = s["table"][b, :-(-n // c["page"])].long()
            k, v = (exact_values(x[at], None if p is None else p[at]).transpose(0, 1).reshape(KV, -1, d)[:, :n] for x, p in ((K, Kp), (V, Vp)))
            for h in range(KV if n else 0):
                rows = slice(h * G, h * G + G)
                out[b, rows] = exact_attention(s["q"][b].double().view(H, d)[rows], k[h], v[h], n)
        return out.view(c["B"], H * d)
    out = torch.zeros(c["T"], H, d, dtype=torch.float64, device="cuda")
    i = j = 0
    for n, m in zip(*prefill_lens(c)):
        for h in range(H):
            q, k, v = s["q"][i:i + n].view(n, H, d)[:, h], s["k"][j:j + m].view(m, KV, d)[:, h // G], s["v"][j:j + m].view(m, KV, d)[:, h // G]
            out[i:i + n, h] = exact_attention(q.double(), k.double(), v.double(), m - n)
        i, j = i + n, j + m
    return out.view(c["T"], H * d)
