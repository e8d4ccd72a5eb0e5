"""Plain 64-bit CPU restatements of the operators that serve drafted tokens."""
import numpy as np
import torch

from tests.serve_ref import BF8, F11, F24


def depths(parent):
    out = []
    for j, p in enumerate(parent):
        assert -1 <= p < j
        out.append(out[p] + 1 if p >= 0 else 0)
    return out


def sees(parent, before):
    """[nodes, before + nodes] bool: what each node of a tree behind `before` tokens sees."""
    n = len(parent)
    m = torch.zeros(n, before + n, dtype=torch.bool)
    m[:, :before] = True
    for j, p in enumerate(parent):
        if p >= 0:
            m[j, before:] = m[p, before:]
        m[j, before + j] = True
    return m


def attend64(q, k, v, see):
    """fp64 attention of q [n, H, d] over k, v [tokens, Hkv, d] (as held), row j over the tokens that
    see [n, tokens] names, with the bound of what f16 weights, fp32 scores and a bf16 output may
    change, per value (derived term by term in serve_ref.attend64)."""
    n, H, d = q.shape
    G = H // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, tol = torch.zeros(n, H, d, dtype=torch.float64), torch.zeros(n, H, d, dtype=torch.float64)
    lse = torch.zeros(H, n, dtype=torch.float64)
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kk.t() / d ** 0.5).masked_fill(~see, -float("inf"))
        p = torch.softmax(s, 1)
        out[:, h] = p @ vv
        mag = (q[:, h].abs() @ kk.abs().t() / d ** 0.5).masked_fill(~see, 0.0).amax(1, keepdim=True)
        es = (d + 6) * F24 * mag * 2 + 2.0 ** -21
        es = es + 2.0 ** -39 * q[:, h].abs().amax(1, keepdim=True) * kk.abs().sum(1).max() / d ** 0.5
        av = p @ vv.abs()
        # (weights of full pages are in units of at most 2^-15 of the largest V step or of 1, the
        # window's step, which counts as one value of 127)
        small = len(kk) * 2.0 ** -38 * max(float(vv.abs().max()), 1.0)
        tol[:, h] = (av * (F11 + 2 * es + 2 * len(kk) * F24) * 1.01 + out[:, h].abs() * BF8 * 1.01 + small
                     + 1e-30)
        lse[h] = torch.logsumexp(s, 1) * 1.4426950408889634
    return out, tol, lse


def probs64(x, temperature):
    """(softmax(x / temperature) in fp64, the bound of what the kernel's fp32 may change).

    Its exponent is (x - max) k: the difference, log2(e), its quotient by the temperature and the
    product round once each, so a weight is off by 4 F24 |x - max| / t and by one step of the
    exponential; the sum by the mean of that and a rounding for each of its additions (a thread's V / 1024
    values and then at most 40 partial sums); its inverse and the product round once each.  What fp32
    cannot hold is below 2^-126."""
    x = x.double().cpu()
    V = x.shape[1]
    t = torch.ones(len(x), dtype=torch.float64) if temperature is None else temperature.double().cpu()
    z = (x - x.amax(1, keepdim=True)) / t[:, None]
    p = torch.softmax(z, 1)
    own = 4 * F24 * torch.where(torch.isinf(z), 0.0, z.abs()) + 2.0 ** -23
    rel = own + (p * own).sum(1, keepdim=True) + (V / 1024 + 42) * F24
    return p, p * rel * 1.01 + 2.0 ** -125


def verify64(token, parent, P, Q, u, u_next, replace):
    """(path, next) of one tree, by the definition, one child after another."""
    P = P.numpy().astype(np.float64)
    Q = None if Q is None else Q.numpy().astype(np.float64)
    V = P.shape[1]
    path = [0]
    while True:
        c = path[-1]
        r, R, Z = P[c].copy(), 1.0, 1.0
        q = None if Q is None else Q[c].copy()
        kept = None
        for j in range(c + 1, len(parent)):
            x = int(token[j])
            if parent[j] != c or not 0 <= x < V:
                continue
            if r[x] > 0 and float(u[j]) * (1.0 if q is None else q[x]) * R < r[x] * Z:
                kept = j
                break
            s = r.copy()
            if q is None:
                s[x] = 0.0
                mass = R - r[x]
            else:
                s = np.maximum(r / R - (q / Z if Z > 0 else 0.0), 0.0)
                mass = s.sum()
            if s.sum() == 0:
                break
            r, R = s, mass
            if q is not None and not replace:
                q[x] = 0.0
                Z = q.sum()
        if kept is None:
            break
        path.append(kept)
    r = np.maximum(r, 0.0)
    total = r.sum()
    if not (total > 0 and np.isfinite(total)):
        return path, -1
    over = np.nonzero(np.cumsum(r) > float(u_next) * total)[0]
    return path, int(over[0]) if len(over) else int(np.nonzero(r)[0][-1])
