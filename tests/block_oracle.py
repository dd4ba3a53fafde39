"""Plain 64-bit forms of the block operators, with bounds on what a correct kernel's results may be off by.  (Not a test module.)

The bounds count roundings: ``u`` is the storage type's unit roundoff (2^-8 for bfloat16, 2^-24 for float32), a sum of n fp32 terms is off by at
most n 2^-24 of the sum of its terms' sizes, and what is rounded to bfloat16 between two products by 2^-8 of itself.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F = 2.0 ** -24


def wide(t):
    return t.detach().double().cpu()


def seen(Tq, Tk, n, m, causal):
    i, j = torch.arange(Tq)[:, None], torch.arange(Tk)
    ok = (i < n) & (j < m)
    return ok & (j - m <= i - n) if causal else ok


def attention(q, k, v, q_lengths=None, k_lengths=None, causal=False, scale=None, do=None):
    """-> {name: (value, bound)} for o and, with do, dq, dk and dv.  Unseen inputs are not touched, whatever they are."""
    dtype = q.dtype
    u, up = U[dtype], (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    q, k, v = wide(q), wide(k), wide(v)
    do = None if do is None else wide(do)
    B, Tq, H, D = q.shape
    Tk, Hkv = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    out = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", k))}
    for b in range(B):
        n = Tq if q_lengths is None else min(max(int(q_lengths[b]), 0), Tq)
        m = Tk if k_lengths is None else min(max(int(k_lengths[b]), 0), Tk)
        ok = seen(Tq, Tk, n, m, causal)[:n, :m]
        if n == 0 or m == 0:
            continue
        for h in range(H):
            g = h // (H // Hkv)
            Q, K, V = q[b, :n, h], k[b, :m, g], v[b, :m, g]
            s = torch.where(ok, scale * Q @ K.T, -math.inf)
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
            p = p / torch.where(p.sum(1, keepdim=True) > 0, p.sum(1, keepdim=True), 1.0)
            # scores: a product of D terms, and a few roundings of their size; twice, for the sum that divides
            es = 2 * torch.where(ok, (D + 8) * F * abs(scale) * (Q.abs() @ K.abs().T), 0.0).amax(1, keepdim=True)
            ep = p * (es + up + (m + 16) * F)
            o = p @ V
            out["o"][0][b, :n, h] = o
            out["o"][1][b, :n, h] = ep @ V.abs() + m * F * (p @ V.abs()) + u * o.abs()
            if do is None:
                continue
            G = do[b, :n, h]
            dp, delta = G @ V.T, (G * o).sum(1, keepdim=True)
            size = (G.abs() * (o.abs())).sum(1, keepdim=True)
            eo = out["o"][1][b, :n, h]
            edelta = (G.abs() * eo).sum(1, keepdim=True) + D * F * size
            ds = p * (dp - delta)
            eds = ep * (dp.abs() + delta.abs()) + p * (D * F * (G.abs() @ V.abs().T) + edelta) + up * ds.abs()
            dq = scale * ds @ K
            out["dq"][0][b, :n, h] = dq
            out["dq"][1][b, :n, h] = abs(scale) * ((eds + m * F * ds.abs()) @ K.abs()) + u * dq.abs()
            terms = n * (H // Hkv) * F
            out["dk"][0][b, :m, g] += scale * ds.T @ Q
            out["dk"][1][b, :m, g] += abs(scale) * ((eds + terms * ds.abs()).T @ Q.abs())
            out["dv"][0][b, :m, g] += p.T @ G
            out["dv"][1][b, :m, g] += (ep + terms * p).T @ G.abs()
    for name in ("dk", "dv"):
        out[name] = (out[name][0], out[name][1] + u * out[name][0].abs())
    return out


def assert_within(got, value, bound, what, slack=1.5):
    """``slack``: the bounds are first-order, and the results of a pass are rounded once more where they are inputs of the next."""
    got = wide(got)
    assert got.shape == value.shape, (what, got.shape, value.shape)
    off = (got - value).abs()
    bad = ~(off <= slack * bound + 1e-30)
    assert not bad.any(), (what, "off by", off[bad].max().item(), "allowed", (slack * bound)[bad].max().item(), "at", bad.nonzero()[0].tolist(), int(bad.sum()))


def norm_rope(x, w, cos, sin, positions, eps, interleaved, dy=None):
    """-> y, or (y, dx, dw), in 64 bits, of x [tokens, heads, D]"""
    x, w = wide(x), wide(w)
    n, rows = 2 * cos.shape[1], cos.shape[0]
    at = positions.cpu().long().clamp(0, rows - 1) if rows else None
    turn = torch.complex(wide(cos), wide(sin))[at][:, None] if n else None
    one = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))

    def rotate(t, back):
        t = t.clone()
        if n:
            z = torch.complex(t[..., one[0]], t[..., one[1]]) * (turn.conj() if back else turn)
            t[..., one[0]], t[..., one[1]] = z.real, z.imag
        return t

    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    y = rotate(x * r * w, False)
    if dy is None:
        return y
    dn = rotate(wide(dy), True)
    g = dn * w
    return y, r * (g - x * r * r * (g * x).mean(-1, keepdim=True)), dn * x * r


def words(n, seed, offset):
    """The generator's first n 16-bit words, one counter at a time in Python's own integers."""
    out, low = [], 0xFFFFFFFF
    for i in range((n + 7) // 8):
        c = [i & low, i >> 32, offset & low, offset >> 32]
        k = [seed & low, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
            k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
        for word in c:
            out += [word & 0xFFFF, word >> 16]
    return torch.tensor(out[:n])
