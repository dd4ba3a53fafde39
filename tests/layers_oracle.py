"""Plain 64-bit forms of layer norm, dense layers and the distillation loss, with bounds on what a correct kernel's results may be off by, counted in
roundings as in block_oracle.py.  (Not a test module.)  Each gives {name: (value, bound)}."""
import math

import torch

from block_oracle import F, U, wide


def layer_norm(x, weight=None, bias=None, residual=None, eps=1e-5, dy=None, ds=None):
    u = U[x.dtype]
    W = x.shape[-1]
    X, dy, ds = (None if t is None else wide(t).reshape(-1, W) for t in (x, dy, ds))
    w, b = (torch.full((W,), v, dtype=torch.float64) if t is None else wide(t) for t, v in ((weight, 1.0), (bias, 0.0)))
    s = X if residual is None else X + wide(residual).reshape(-1, W)
    mean = s.mean(1, keepdim=True)
    d = s - mean
    r = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    n = d * r
    # the mean is a sum of W terms; every difference from it has its error, and roundings of its own
    emean = (W + 2) * F * s.abs().mean(1, keepdim=True)
    ed = emean + 2 * F * (s.abs() + d.abs())
    er = (W + 8) * F + (d.abs() * ed).mean(1, keepdim=True) * r.square()            # relative
    en = r * ed + n.abs() * (er + 2 * F)
    y = n * w + b
    out = {"y": (y, w.abs() * en + 3 * F * ((n * w).abs() + b.abs()) + u * y.abs())}
    if residual is not None:
        out["s"] = (s, u * s.abs())
    if dy is not None:
        # what was normed comes back rounded
        eu = r * (ed + (u * s.abs() if residual is not None else 0.0) + 2 * F * (s.abs() + mean.abs())) + n.abs() * (er + 2 * F)
        g = dy * w
        mg, mgu = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
        emg = (W + 4) * F * g.abs().mean(1, keepdim=True)
        emgu = (g.abs() * eu).mean(1, keepdim=True) + (W + 4) * F * (g * n).abs().mean(1, keepdim=True)
        dx = r * (g - mg - n * mgu)
        size = g.abs() + mg.abs() + (n * mgu).abs()
        edx = r * (emg + n.abs() * emgu + eu * mgu.abs() + 4 * F * size) + er * r * size
        if ds is not None:
            dx, edx = dx + ds, edx + F * ds.abs()
        terms = len(s) + 4
        dw, db = (dy * n).sum(0), dy.sum(0)
        out["dx"] = (dx, edx + u * dx.abs())
        out["dweight"] = (dw, (dy.abs() * eu).sum(0) + terms * F * (dy * n).abs().sum(0) + u * dw.abs())
        out["dbias"] = (db, terms * F * dy.abs().sum(0) + u * db.abs())
    return {k: (v.reshape(x.shape) if v.dim() == 2 else v, e.reshape(x.shape) if e.dim() == 2 else e) for k, (v, e) in out.items()}


def activation(name, z, precise):
    """-> act(z), act'(z) and bounds of the errors of each as evaluated in fp32, at z itself."""
    if name is None:
        return z, torch.ones_like(z), 0 * z, 0 * z
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), 0 * z, 0 * z
    if name == "gelu":
        gate, rise = 0.5 * torch.special.erfc(-z / math.sqrt(2)), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        # the fit's own error, and that of the exponential, whose argument is z^2 / 2
        rel = (4.1e-7 if precise else 4.7e-6) + (4 + 2 * z * z) * F
    else:
        a = math.sqrt(2 / math.pi)
        arg, slope = (z, 1.0) if name == "silu" else (2 * a * (z + 0.044715 * z ** 3), 2 * a * (1 + 3 * 0.044715 * z * z))
        gate = torch.sigmoid(arg)
        rise = gate * torch.sigmoid(-arg) * slope
        rel = (6 + 4 * arg.abs()) * F
    tail = torch.minimum(gate, 1 - gate)
    y, dy = z * gate, gate + z * rise
    return y, dy, z.abs() * tail * rel + 4 * F * y.abs(), rel * (tail + (z * rise).abs()) + 8 * F * (gate + (z * rise).abs())


def linear(x, weight, bias=None, residual=None, act=None, dy=None):
    u, precise = U[x.dtype], x.dtype == torch.float32
    X, w = wide(x).reshape(-1, x.shape[-1]), wide(weight)
    O, I = w.shape
    T = len(X)
    b = torch.zeros(O, dtype=torch.float64) if bias is None else wide(bias)
    res = 0.0 if residual is None else wide(residual).reshape(T, O)
    z = X @ w.T + b
    ez = (I + 2) * F * (X.abs() @ w.abs().T + b.abs())
    a, slope, ea, eslope = activation(act, z, precise)
    y = a + res
    # no activation is steeper than 1.2
    out = {"y": (y, 1.2 * ez + ea + 2 * F * (a.abs() + (res.abs() if residual is not None else 0.0)) + u * y.abs())}
    if dy is not None:
        g = wide(dy).reshape(T, O)
        dz = g * slope
        if act is None:
            edz = erounded = 0 * g
        else:
            # what goes into the activation comes back rounded; no second derivative is above 1, but relu's slope jumps
            off = ez + u * z.abs()
            jump = (z.abs() <= 2 * off).double() if act == "relu" else off
            edz = g.abs() * (jump + eslope) + F * dz.abs()
            erounded = edz + u * dz.abs()
        dx, dw, db = dz @ w, dz.T @ X, dz.sum(0)
        out["dx"] = (dx, erounded @ w.abs() + (O + 2) * F * (dz.abs() @ w.abs()) + u * dx.abs())
        out["dweight"] = (dw, erounded.T @ X.abs() + (T + 2) * F * (dz.abs().T @ X.abs()) + u * dw.abs())
        out["dbias"] = (db, edz.sum(0) + (T + 4) * F * dz.abs().sum(0) + u * db.abs())
        out["dresidual"] = (g.reshape(dy.shape), 0 * g.reshape(dy.shape))
    lead = x.shape[:-1]
    return {k: (v.reshape(*lead, -1), e.reshape(*lead, -1)) if k in ("y", "dx") else (v, e) for k, (v, e) in out.items()}


def distill(logits, teacher, ids, labels=None, temperature=1.0, label_weight=0.0, dloss=None):
    """One row after the other, as the definition has it."""
    u, tau, lw = U[logits.dtype], temperature, label_weight
    V = logits.shape[-1]
    Z = wide(logits).reshape(-1, V)
    T, C = wide(teacher).reshape(len(Z), -1) if teacher.numel() else wide(teacher).new_zeros(len(Z), 0), ids.cpu().reshape(len(Z), ids.shape[-1])
    L = None if labels is None else labels.cpu().reshape(-1)
    G = None if dloss is None else wide(dloss).reshape(-1)
    loss, eloss = torch.zeros(len(Z), dtype=torch.float64), torch.zeros(len(Z), dtype=torch.float64)
    dz, edz = torch.zeros_like(Z), torch.zeros_like(Z)

    def softmax(z, t):
        """Probabilities, their logarithms and the relative error of the sum that divides: sums of a lane and over lanes, arguments rounded."""
        top = z.max()
        arg = (z - top) / t
        total = torch.exp(arg).sum()
        q = torch.exp(arg) / total
        finite = torch.where(q > 0, arg.abs(), 0.0)
        return q, arg - total.log(), (V / 64 + 64) * F + (q * finite * 3 * F).sum(), (finite * 3 + 4) * F

    for i, z in enumerate(Z):
        keep = (C[i] >= 0) & (C[i] < V) & (T[i] != -math.inf)
        c, t = C[i][keep].long(), T[i][keep]
        label = -1 if L is None else int(L[i])
        label = label if 0 <= label < V and lw > 0 else -1
        if len(c) > 0 and lw < 1:
            q, logq, es, eq = softmax(z, tau)
            arg = (t - t.max()) / tau
            p = torch.exp(arg) / torch.exp(arg).sum()
            logp = arg - torch.exp(arg).sum().log()
            some = p > 0
            ep = p * ((len(c) + 8) * F + torch.where(some, arg.abs(), 0.0) * 3 * F + (p * torch.where(some, arg.abs(), 0.0) * 3 * F).sum())
            terms = torch.where(some, p * (logp - logq[c]), 0.0)
            scale = (1 - lw) * tau * tau
            loss[i] += scale * terms.sum()
            eloss[i] += scale * (es + 8 * F + (ep[some] * ((logp - logq[c])[some].abs() + 1)).sum())
            if G is not None:
                k = G[i] * (1 - lw) * tau
                e = k.abs() * q * (es + eq)
                d = k * q
                d.index_add_(0, c, -k * p)
                e.index_add_(0, c, k.abs() * (ep + 4 * F * p))
                dz[i] += d
                edz[i] += e + 6 * F * k.abs() * q
        if label >= 0:
            q, logq, es, eq = softmax(z, 1.0)
            loss[i] -= lw * logq[label]
            eloss[i] += lw * (es + 8 * F)
            if G is not None:
                k = G[i] * lw
                right = torch.zeros(V, dtype=torch.float64)
                right[label] = 1.0
                dz[i] += k * (q - right)
                edz[i] += k.abs() * (q * (es + eq + 6 * F) + 4 * F * right)
    out = {"loss": (loss.reshape(logits.shape[:-1]), (eloss + F * loss.abs()).reshape(logits.shape[:-1]))}
    if G is not None:
        out["dlogits"] = (dz.reshape(logits.shape), (edz + u * dz.abs()).reshape(logits.shape))
    return out
