"""The work that the softmax attention of a transformer's other layers is measured on.

A case is one attention layer; its `op` says which part of a program it stands for:
  train    forward and gradients: O, dQ, dK, dV and, with a position bias, the gradient of its table
  infer    the forward pass alone: O
  serve    a few new tokens of every sequence over a cache, behind a prefix that all sequences share
           or behind none: O
Q is [B, H, Nq, d], K and V are [B, H / G, Nk, d] (every K, V head serves G query heads), or with the
two middle axes swapped where `layout` is "token"; "fused" tensors are the slices of one projection output.
A ragged batch keeps lengths per sequence, and what lies behind a length is not read: rows behind a
sequence's queries come back as zeros.  The position bias is table[bucket(key position - query position), head].
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _case(name, op, dtype, B, H, G, d, Nq, Nk, causal=False, ragged=False, buckets=0, far=128, two_sided=False,
          prefix=0, layout="head"):
    c = {"op": op, "dtype": dtype, "B": B, "H": H, "G": G, "d": d, "Nq": Nq, "Nk": Nk, "causal": causal,
         "ragged": ragged, "buckets": buckets, "far": far, "two_sided": two_sided, "prefix": prefix, "layout": layout}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest calls: a test-sized float layer with an odd number of keys
        _case("tiny_cross_fp32_train", "train", "fp32", 1, 2, 1, 64, 100, 37),
        # a short clip in float (gradient checks, float reference runs): 5 x 30 x 13 latents
        _case("clip_fp32_train", "train", "fp32", 1, 4, 1, 128, 1950, 1950),
        # cross attention of a video layer to the tokens of two prompts of different lengths
        _case("cross_video_train", "train", "bf16", 2, 12, 1, 128, 32760, 512, ragged=True, layout="token"),
        # the layer of an image model that is kept dense: 32 x 32 latents, slices of the fused projection
        _case("image_dense_train", "train", "bf16", 16, 16, 1, 64, 1024, 1024, layout="fused"),
        # a causal layer with four query heads per K, V head
        _case("causal_shared_heads_train", "train", "bf16", 2, 16, 4, 128, 4096, 4096, causal=True),
        # a text encoder: ragged prompts, learned bias in 32 two-sided buckets
        _case("text_bias_train", "train", "bf16", 8, 12, 1, 64, 512, 512, ragged=True, buckets=32, two_sided=True),
        # a longer causal sequence (odd length) with the one-sided bias, sampled
        _case("causal_bias_infer", "infer", "bf16", 1, 12, 1, 64, 5001, 5001, causal=True, buckets=32),
        # the video layer kept dense: 12 heads, 21 x 30 x 52 latents
        _case("video_dense_train", "train", "bf16", 1, 12, 1, 128, 32760, 32760),
        # one sequence, one new token: latency
        _case("token_one", "serve", "bf16", 1, 12, 1, 128, 1, 1000, causal=True),
        # a full batch, one new token each, ragged caches
        _case("token_batch", "serve", "bf16", 16, 32, 4, 128, 1, 8192, causal=True, ragged=True, layout="token"),
        # many continuations of one long prompt, one new token each
        _case("prefix_batch", "serve", "bf16", 32, 16, 4, 128, 1, 700, causal=True, ragged=True, prefix=16384),
        # a few new tokens at a time behind a shared prompt of odd length, with the one-sided bias
        _case("prefix_chunk_bias", "serve", "bf16", 6, 12, 1, 64, 7, 259, causal=True, ragged=True, buckets=32,
              prefix=2111),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    limit = {c["op"]: 0 for c in listed()}
    for c in listed():
        limit[c["op"]] = max(limit[c["op"]], work(c)["flops"])
    while True:
        op = rng.choice(("train", "train", "infer", "serve", "serve"))
        fp32 = rng.random() < 0.2
        d = rng.choice((64, 128))
        G = rng.choice((1, 1, 2, 4))
        B, H = rng.choice((1, 1, 2, 4, 8)), G * _log_uniform(rng, 1, 16)
        buckets = rng.choice((0, 0, 0, 16, 32))
        two_sided = rng.random() < 0.5
        far = rng.choice((64, 128, 256))
        if op == "serve":
            B = _log_uniform(rng, 1, 32)
            prefix = rng.choice((0, _log_uniform(rng, 64, 20000)))
            c = _case(None, op, "fp32" if fp32 else "bf16", B, H, G, d, rng.choice((1, 1, 1, 2, 5, 8)),
                      _log_uniform(rng, 16, 1500 if prefix else 16000), True, rng.random() < 0.7, buckets, far, False, prefix,
                      rng.choice(("head", "token")))
        else:
            n = _log_uniform(rng, 40, 3000 if fp32 else 24000)
            self_attention = buckets > 0 or rng.random() < 0.6
            m = n if self_attention else _log_uniform(rng, 1, 2000)
            causal = self_attention and rng.random() < 0.5
            layouts = ("head", "token", "fused") if self_attention and G == 1 else ("head", "token")
            c = _case(None, op, "fp32" if fp32 else "bf16", B, H, G, d, n, m, causal, B > 1 and rng.random() < 0.5, buckets,
                      far, two_sided and not causal, 0, rng.choice(layouts))
        elements = c["B"] * max(c["H"] * c["Nq"], c["H"] // c["G"] * c["Nk"]) * d
        # (a float product takes about eight times as long as a bf16 one)
        if elements <= 1 << 28 and work(c)["flops"] * (8 if fp32 else 1) <= max(limit[op], limit["train"] // 20):
            return c


# ---------------------------------------------------------------- inputs

def _lengths(c):
    """(queries, keys) of every sequence.  A ragged batch goes from full length down to a fifth of it; a
    serving batch down to a sequence that holds nothing but its new tokens."""
    B, Nq, Nk = c["B"], c["Nq"], c["Nk"]
    if not c["ragged"]:
        return [Nq] * B, [Nk] * B
    share = [1.0 - 0.8 * b / max(1, B - 1) for b in range(B)]
    k = [max(min(Nq, Nk) if c["op"] == "serve" else 1, round(Nk * s)) for s in share]
    if c["op"] == "serve":
        if B > 1:
            k[-1] = min(Nq, Nk)
        return [Nq] * B, k
    return (k if Nq == Nk else [Nq] * B), k


def _q_pos(c):
    """Position of the first query of every sequence."""
    if c["op"] == "serve":
        return [c["prefix"] + k - c["Nq"] for k in _lengths(c)[1]]
    return [c["Nk"] - c["Nq"]] * c["B"]


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    B, H, G, d, Nq, Nk, dt = c["B"], c["H"], c["G"], c["d"], c["Nq"], c["Nk"], _DTYPES[c["dtype"]]
    Hk = H // G
    token = c["layout"] != "head"

    def tensor(heads, n):
        shape = (B, n, heads, d) if token else (B, heads, n, d)
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(dt)

    s = {"case": c}
    if c["layout"] == "fused":
        qkv = torch.stack([tensor(H, Nq) for _ in range(3)], dim=2)
        s["Q"], s["K"], s["V"] = (qkv[:, :, i] for i in range(3))
    else:
        s["Q"], s["K"], s["V"] = tensor(H, Nq), tensor(Hk, Nk), tensor(Hk, Nk)
    if c["prefix"]:
        s["prefix"] = tuple(
            torch.randn((c["prefix"], Hk, d) if token else (Hk, c["prefix"], d), generator=gen, device=dev).to(dt)
            for _ in range(2))
    s["table"] = None
    if c["buckets"]:
        s["table"] = torch.randn(c["buckets"], H, generator=gen, device=dev).to(dt)
    if c["op"] == "train":
        s["dO"] = tensor(H, Nq)
        for k in ("Q", "K", "V", "table"):
            if s[k] is not None:
                s[k] = s[k].detach().requires_grad_(True)
    q_len, k_len = _lengths(c)
    as_ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    s["q_len"], s["k_len"], s["q_pos"] = as_ints(q_len), as_ints(k_len), as_ints(_q_pos(c))
    if own:
        from paper_2509_24006_amd import autograd as attn
        s["attn"] = attn
        s["buckets"] = attn.position_buckets(c["buckets"], c["far"], c["two_sided"]) if c["buckets"] else None
    elif c["buckets"]:
        s["borders"] = torch.tensor(_borders(c), device=dev)
    return s


# ---------------------------------------------------------------- a pass

def run(state):
    if not own:
        return _plain(state)
    s, c = state, state["case"]
    token = c["layout"] != "head"
    ragged = c["ragged"]
    if c["op"] == "serve":
        with torch.no_grad():
            return s["attn"].cached_attention(s["Q"], s["K"], s["V"], k_len=s["k_len"] if ragged else None,
                                              prefix=s.get("prefix"), causal=c["causal"], table=s["table"],
                                              buckets=s["buckets"], token_major=token)
    given = dict(causal=c["causal"], q_len=s["q_len"] if ragged and c["Nq"] == c["Nk"] else None,
                 k_len=s["k_len"] if ragged else None, table=s["table"], buckets=s["buckets"], token_major=token)
    if c["op"] == "infer":
        with torch.no_grad():
            return s["attn"].dense_attention(s["Q"], s["K"], s["V"], **given)
    O = s["attn"].dense_attention(s["Q"], s["K"], s["V"], **given)
    leaves = [s[k] for k in ("Q", "K", "V", "table") if s[k] is not None]
    return (O,) + torch.autograd.grad(O, leaves, s["dO"])


# ---------------------------------------------------------------- the plain form

def _borders(c):
    """Distances at which a new bucket begins.  Of the `half` buckets of a side the first half // 2 hold one distance
    each, and the others grow by a constant factor up to `far`: bucket e + k begins at e (far / e)^(k / (half - e)),
    found in whole numbers."""
    half = c["buckets"] // 2 if c["two_sided"] else c["buckets"]
    e = half // 2
    m = half - e
    out = list(range(1, e + 1))
    for k in range(1, m):
        n = out[-1]
        while n ** m < c["far"] ** k * e ** (m - k):
            n += 1
        out.append(n)
    return out


_CHUNK = 1 << 27                  # scores that are formed at a time


def _plain(s):
    c = s["case"]
    B, H, G, d, Nq, prefix = c["B"], c["H"], c["G"], c["d"], c["Nq"], c["prefix"]
    token, train = c["layout"] != "head", c["op"] == "train"
    dev, scale = s["Q"].device, 1.0 / math.sqrt(d)
    heads = lambda x: x.detach().transpose(1, 2) if token else x.detach()
    Q, K, V = heads(s["Q"]), heads(s["K"]), heads(s["V"])
    O = torch.zeros_like(s["Q"], memory_format=torch.contiguous_format)
    Oh = heads(O)
    if train:
        dO = heads(s["dO"])
        grads = [torch.zeros_like(s[k], memory_format=torch.contiguous_format) for k in ("Q", "K", "V")]
        dQh, dKh, dVh = (heads(x) for x in grads)
        dT = torch.zeros(c["buckets"], H, dtype=torch.float64, device=dev) if c["buckets"] else None
    shared = [(x.transpose(0, 1) if token else x) for x in s.get("prefix", ())]
    q_len, k_len = _lengths(c)
    q_pos = _q_pos(c)
    table = s["table"].detach().float() if s["table"] is not None else None
    for b in range(B):
        nq, nk = (q_len[b] if Nq == c["Nk"] and c["op"] != "serve" else Nq), k_len[b] + prefix
        kb, vb = K[b, :, :k_len[b]].float(), V[b, :, :k_len[b]].float()
        if prefix:
            kb, vb = torch.cat([shared[0].float(), kb], 1), torch.cat([shared[1].float(), vb], 1)
        rows = max(1, min(nq, _CHUNK // nk))
        step = max(1, min(H // G, _CHUNK // (rows * nk * G)))
        keys = torch.arange(nk, device=dev)
        for h in range(0, H // G, step):
            g = min(H // G, h + step) - h
            k, v = kb[h:h + g], vb[h:h + g]
            kt, vt = k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
            if train:
                dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            for u in range(G):                       # the u-th query head of every K, V head
                hq = torch.arange(h, h + g, device=dev) * G + u
                for r in range(0, nq, rows):
                    e = min(nq, r + rows)
                    q = Q[b, hq, r:e].float()
                    S = torch.matmul(q, kt).mul_(scale)
                    rel = keys - (q_pos[b] + torch.arange(r, e, device=dev)).unsqueeze(1)
                    if table is not None:
                        S += table.T[hq][:, _bucket(rel, s["borders"], c["two_sided"])]
                    if c["causal"]:
                        S.masked_fill_(rel > 0, -math.inf)
                    m = S.amax(2, keepdim=True)
                    P = torch.exp(S.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)))
                    l = P.sum(2, keepdim=True)
                    P /= torch.where(l > 0, l, torch.ones_like(l))
                    Oh[b, hq, r:e] = torch.matmul(P, v).to(O.dtype)
                    if not train:
                        continue
                    do = dO[b, hq, r:e].float()
                    dv += torch.matmul(P.transpose(1, 2).contiguous(), do)
                    dS = torch.matmul(do, vt)
                    dS = P * (dS - (P * dS).sum(2, keepdim=True))
                    dQh[b, hq, r:e] = (torch.matmul(dS, k) * scale).to(O.dtype)
                    dk += torch.matmul(dS.transpose(1, 2).contiguous(), q)
                    if table is not None:
                        # sums along the diagonals (rows pushed against each other by one column), then by bucket
                        n = e - r
                        skew = torch.nn.functional.pad(dS.flip(1), (0, n)).view(g, -1)[:, :n * (nk + n - 1)]
                        diag = skew.view(g, n, nk + n - 1).sum(1, dtype=torch.float64)
                        off = torch.arange(nk + n - 1, device=dev) - (n - 1) - (q_pos[b] + r)
                        of = _bucket(off, s["borders"], c["two_sided"])
                        hot = (of.unsqueeze(0) == torch.arange(c["buckets"], device=dev).unsqueeze(1)).double()
                        dT[:, hq] += torch.matmul(hot, diag.T.contiguous())
            if train:
                dKh[b, h:h + g, :k_len[b]] = (dk * scale).to(O.dtype)
                dVh[b, h:h + g, :k_len[b]] = dv.to(O.dtype)
    if not train:
        return O
    return (O, *grads) + ((dT.to(s["table"].dtype),) if c["buckets"] else ())


def _bucket(rel, borders, two_sided):
    n = rel.abs() if two_sided else (-rel).clamp(min=0)
    u = torch.bucketize(n, borders, right=True)
    return u + (rel > 0) * (len(borders) + 1) if two_sided else u


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Inputs up to their lengths read once and outputs written once; operations of the pairs that the
    masks leave (4 d forward, 10 d backward), the products of the backward pass counted once each."""
    c = case
    B, H, G, d, Nq, Nk, prefix = c["B"], c["H"], c["G"], c["d"], c["Nq"], c["Nk"], c["prefix"]
    esz = 2 if c["dtype"] == "bf16" else 4
    q_len, k_len = _lengths(c)
    pairs = keys = rows = 0
    for b in range(B):
        nq = q_len[b] if Nq == Nk and c["op"] != "serve" else Nq
        total = k_len[b] + prefix
        rows += nq
        keys += k_len[b]
        if not c["causal"]:
            pairs += nq * total
        else:
            first = _q_pos(c)[b] + 1                       # keys that the first query sees
            full = min(nq, max(0, total - first))          # rows before the one that sees them all
            pairs += full * first + full * (full - 1) // 2 + (nq - full) * total
    train = c["op"] == "train"
    q_bytes, kv_bytes = H * rows * d * esz, H // G * keys * d * esz
    out_rows = H * B * Nq * d * esz
    nbytes = q_bytes + 2 * kv_bytes + out_rows + 2 * (H // G) * prefix * d * esz + c["buckets"] * H * esz
    if train:
        nbytes += q_bytes + out_rows + 2 * H // G * B * Nk * d * esz + c["buckets"] * H * esz
    return {"bytes": nbytes, "flops": (14 if train else 4) * H * pairs * d}


# ---------------------------------------------------------------- the same layer in 64 bits

def _bucket_of(distance, half, far):
    """The largest bucket of a side that begins at or below this distance, from its definition."""
    e = half // 2
    if distance < e:
        return distance
    m, k = half - e, 0
    while k < m - 1 and distance ** m * e ** (k + 1) >= far ** (k + 1) * e ** m:
        k += 1
    return e + k


def exact(case, seed):
    """Softmax attention head by head in float64 with torch's own derivatives; the bias is looked up in a list
    of buckets over all offsets."""
    c = case
    pairs = c["B"] * c["H"] * c["Nq"] * (c["Nk"] + c["prefix"])
    if pairs > (1 << 30 if c["buckets"] else 1 << 34):
        return None
    s = prepare(c, seed)
    dev, train, token = s["Q"].device, c["op"] == "train", c["layout"] != "head"
    B, H, G, d, Nq, Nk, prefix = c["B"], c["H"], c["G"], c["d"], c["Nq"], c["Nk"], c["prefix"]
    at = (lambda x, b, h: x[b, :, h]) if token else (lambda x, b, h: x[b, h])
    wide = {k: s[k].detach().double() for k in ("Q", "K", "V")}
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device=dev)
    grads = {k: torch.zeros(s[k].shape, dtype=torch.float64, device=dev) for k in ("Q", "K", "V")} if train else {}
    q_len, k_len = _lengths(c)
    q_pos = _q_pos(c)
    table = s["table"].detach().double().requires_grad_(train) if c["buckets"] else None
    if c["buckets"]:
        half = c["buckets"] // 2 if c["two_sided"] else c["buckets"]
        reach = prefix + Nk + Nq
        names = []
        for off in range(-reach, reach + 1):
            n = abs(off) if c["two_sided"] else max(-off, 0)
            names.append(_bucket_of(min(n, c["far"]), half, c["far"]) + (half if c["two_sided"] and off > 0 else 0))
        names = torch.tensor(names, device=dev)
    for b in range(B):
        nq = q_len[b] if Nq == Nk and c["op"] != "serve" else Nq
        for h in range(H):
            k, v = (at(wide[x], b, h // G)[:k_len[b]].requires_grad_(train) for x in ("K", "V"))
            kk, vv = k, v
            if prefix:
                pick = (lambda x: x[:, h // G]) if token else (lambda x: x[h // G])
                kk, vv = (torch.cat([pick(x).double(), y]) for x, y in zip(s["prefix"], (k, v)))
            for r in range(0, nq, 8192):
                e = min(nq, r + 8192)
                q = at(wide["Q"], b, h)[r:e].requires_grad_(train)
                score = (q @ kk.T) / math.sqrt(d)
                off = torch.arange(len(kk), device=dev)[None] - torch.arange(r, e, device=dev)[:, None] - q_pos[b]
                if c["buckets"]:
                        score = score + table[:, h][names[off + reach]]
                if c["causal"]:
                    score = score.masked_fill(off > 0, -math.inf)
                seen = (score > -math.inf).any(1, keepdim=True)
                p = torch.softmax(torch.where(seen, score, torch.zeros_like(score)), 1) * seen
                o = p @ vv
                at(O, b, h)[r:e] = o.detach()
                if train:
                    o.backward(at(s["dO"], b, h)[r:e].double())
                    at(grads["Q"], b, h)[r:e] = q.grad
            if train:
                at(grads["K"], b, h // G)[:k_len[b]] += k.grad
                at(grads["V"], b, h // G)[:k_len[b]] += v.grad
    if not train:
        return O
    return (O, grads["Q"], grads["K"], grads["V"]) + ((table.grad,) if c["buckets"] else ())
