"""Softmax attention in 64 bits from its formulas, with a bound for every element of what the library may return.

u is half a step of the tensors' type (relative), e half a step of float.  The library rounds to the tensors' type: P
where it enters a product, dS where it enters a product, and every result.  Its O enters D = rowsum(dO O).  All other
arithmetic is in float: a dot product of n terms is off by at most n e times the sum of their magnitudes, and
an exponential by the error of its argument and a few steps of its own."""
import torch

E32 = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def bucket(rel, buckets, two_sided):
    """buckets: ascending borders"""
    n = rel.abs() if two_sided else (-rel).clamp(min=0)
    u = sum((n >= x).long() for x in buckets) if buckets else torch.zeros_like(n)
    return u + (rel > 0).long() * (len(buckets) + 1) if two_sided else u


def attention(Q, K, V, scale, causal=False, q_len=None, k_len=None, pos=None, table=None, borders=(), two_sided=False,
              prefix=None, dO=None, result=torch.bfloat16):
    """Q [B,H,Nq,d], K, V [B,Hkv,Nk,d], prefix (K, V) [Hkv,Np,d]; pos: position of the first query per sequence.  Returns
    {name: (value, bound)} in float64 for O, L and, with dO, dQ, dK, dV, dtable."""
    dev, (B, H, Nq, d), (Hkv, Nk) = Q.device, Q.shape, K.shape[1:3]
    G, u = H // Hkv, U[result]
    Np = 0 if prefix is None else prefix[0].shape[1]
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)
    out = {"O": (z(B, H, Nq, d), z(B, H, Nq, d)), "L": (z(B, H, Nq), z(B, H, Nq))}
    if dO is not None:
        for n, s in (("dQ", (B, H, Nq, d)), ("dK", (B, Hkv, Nk, d)), ("dV", (B, Hkv, Nk, d))):
            out[n] = (z(*s), z(*s))
        if table is not None:
            out["dtable"] = (z(*table.shape), z(*table.shape))
    for b in range(B):
        nq = Nq if q_len is None else min(max(int(q_len[b]), 0), Nq)
        nk = Nk if k_len is None else min(max(int(k_len[b]), 0), Nk)
        p0 = int(pos[b])
        for h in range(H):
            hk = h // G
            q, k, v = Q[b, h, :nq].double(), K[b, hk, :nk].double(), V[b, hk, :nk].double()
            if Np:
                k, v = torch.cat([prefix[0][hk].double(), k]), torch.cat([prefix[1][hk].double(), v])
            rel = torch.arange(len(k), device=dev)[None] - torch.arange(nq, device=dev)[:, None] - p0
            seen = rel <= 0 if causal else torch.ones_like(rel, dtype=torch.bool)
            S = (q @ k.T) * scale
            mag = (q.abs() @ k.abs().T) * scale * (d + 2)     # times e: error of the float scores
            if table is not None:
                bk = bucket(rel, list(borders), two_sided)
                t = table.double()[:, h][bk]
                seen = seen & (t > -1e30)                     # (lower entries hide their pairs)
                t = torch.where(seen, t, torch.zeros_like(t))
                S = S + t
                mag = mag + 2 * t.abs()
            S = S.masked_fill(~seen, -torch.inf)
            L = torch.logsumexp(S, 1, keepdim=True)
            some = seen.any(1, keepdim=True)
            P = torch.exp(S - torch.where(some, L, torch.zeros_like(L))).masked_fill(~seen, 0.0)
            # relative error of a probability in float: its score, the sum, the statistics
            top = torch.where(seen, mag, torch.zeros_like(mag)).amax(1, keepdim=True) if len(k) and nq else torch.zeros_like(L)
            size = torch.where(some, L, torch.zeros_like(L)).abs() + torch.where(seen, S, torch.zeros_like(S)).abs()
            f = E32 * (mag + top + 3 * size + len(k) + 32)
            O = P @ v
            tO = u * O.abs() + (P * (u + 2 * f + E32 * len(k))) @ v.abs()
            out["O"][0][b, h, :nq], out["O"][1][b, h, :nq] = O, tO
            out["L"][0][b, h] = -torch.inf
            out["L"][0][b, h, :nq] = torch.where(some, L, torch.full_like(L, -torch.inf))[:, 0]
            out["L"][1][b, h, :nq] = (E32 * (top + 4 * L.abs().nan_to_num(0, 0, 0) + len(k) + 32))[:, 0]
            if dO is None:
                continue
            g = dO[b, h, :nq].double()
            tD = (g.abs() * (tO + E32 * (d + 2) * O.abs())).sum(1, keepdim=True)
            dP, D = g @ v.T, (g * O).sum(1, keepdim=True)
            dS = P * (dP - D)
            tS0 = 3 * f * dS.abs() + P * (tD + E32 * (d + 2) * (g.abs() @ v.abs().T) + 2 * E32 * D.abs())   # in float
            tS = tS0 + u * (dS.abs() + tS0)
            out["dQ"][0][b, h, :nq] = scale * (dS @ k)
            out["dQ"][1][b, h, :nq] = u * (scale * (dS @ k)).abs() + 1.01 * scale * ((tS + E32 * len(k) * dS.abs()) @ k.abs())
            n = G * nq
            dv, dk = P.T @ g, scale * (dS.T @ q)
            out["dV"][0][b, hk, :nk] += dv
            out["dK"][0][b, hk, :nk] += dk
            out["dV"][1][b, hk, :nk] += 1.01 * (P * (u + 2 * f + E32 * n)).T @ g.abs()
            out["dK"][1][b, hk, :nk] += 1.01 * scale * ((tS + E32 * n * dS.abs()).T @ q.abs())
            if table is not None:
                # (sums over all sequences: n terms of float additions in any order)
                m = dS.numel() * B
                for x, y in ((out["dtable"][0], dS), (out["dtable"][1], tS0 + E32 * m * dS.abs())):
                    x[:, h].index_add_(0, bk.reshape(-1), y.reshape(-1))
    if dO is not None:
        for n in ("dK", "dV"):
            out[n][1].add_(u * out[n][0].abs())
        if table is not None:
            out["dtable"][1].add_(U[table.dtype] * out["dtable"][0].abs())
    return out
