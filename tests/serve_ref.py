"""Plain 64-bit (and, where codes must match bit for bit, fp32-ordered) CPU
restatements of the serving operators, and the cache's layouts as index maps."""
import numpy as np
import torch

F24 = 2.0 ** -24                # half a step of fp32, relative
BF8 = 2.0 ** -8                 # half a step of bf16, relative
F11 = 2.0 ** -11                # half a step of fp16, relative


def f64(t):
    return t.detach().cpu().double()


def norm64(X, R, gain, bias, eps):
    """(H in X's dtype, y in fp64, y without the shift in fp64)."""
    H = X.cpu() if R is None else (X.cpu().float() + R.cpu().float()).to(X.dtype)
    h = H.double()
    y0 = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gain.cpu().double()
    return H, (y0 if bias is None else y0 + bias.cpu().double()), y0


def linear64(codes, h, z, w, h_w, z_w, B):
    a = f64(codes) - f64(z)[:, None]
    b = f64(w) - f64(z_w).reshape(-1, 1)
    y = (a @ b.t()) * f64(h)[:, None] * f64(h_w).reshape(1, -1)
    return y if B is None else y + f64(B)


# ------------------------------------------------------------------ the cache, kept as plain rows
def quant_block(x):
    """x fp32 [page, d] of one head -> (codes fp32, step): the fp32 order of the symmetric quantiser."""
    x = x.numpy().astype(np.float32)
    a = np.abs(x).max()
    if not np.isfinite(x).all():
        return torch.zeros(x.shape), float("nan")
    h = max(np.float32(a / np.float32(127.0)), np.float32(1e-5))
    q = np.clip(np.rint(x * np.float32(np.float32(1.0) / h)), -127, 127)
    return torch.from_numpy(q), float(h)


def turn32(x, cs, sn):
    """RoPE in the block step's fp32 order: x [n, heads, d], cs, sn [n, 1, d / 2]."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)


class PlainCache:
    """One sequence's keys or values as bf16 rows [tokens, kv_heads, d]."""

    def __init__(self, page, kv_heads, d):
        self.page, self.rows = page, torch.zeros(0, kv_heads, d, dtype=torch.bfloat16)

    def add(self, rows):
        self.rows = torch.cat([self.rows, rows])

    def values(self):
        """The rows as the cache stands for them, fp32: full pages through their codes."""
        out = self.rows.float().clone()
        P = self.page
        for p in range(len(out) // P):
            for u in range(out.shape[1]):
                q, h = quant_block(out[p * P:(p + 1) * P, u])
                out[p * P:(p + 1) * P, u] = q * torch.tensor(h, dtype=torch.float32)
        return out


def attend64(q, k, v, before):
    """fp64 attention of one sequence: q [n, H, d], k, v [tokens, Hkv, d] (as held), with the
    bound of what f16 weights, fp32 scores and a bf16 output may change, per value."""
    n, H, d = q.shape
    G = H // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, tol = torch.zeros(n, H, d, dtype=torch.float64), torch.zeros(n, H, d, dtype=torch.float64)
    lse = torch.zeros(H, n, dtype=torch.float64)
    hide = torch.arange(len(k)) > (before + torch.arange(n))[:, None]
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kk.t() / d ** 0.5).masked_fill(hide, -float("inf"))
        p = torch.softmax(s, 1)
        out[:, h] = p @ vv
        # a score is d exact products summed in fp32, times two fp32 factors, minus the maximum:
        # each step is off by half a unit of what it holds, in the exponent
        mag = (q[:, h].abs() @ kk.abs().t() / d ** 0.5).masked_fill(hide, 0.0).amax(1, keepdim=True)
        es = (d + 6) * F24 * mag * 2 + 2.0 ** -21
        # prompts' queries enter as f16 of at least 2^14 at the row's largest entry: bf16's 8 bits fit
        # f16's 11, and an entry that falls below f16's smallest step, 2^-24, loses at most half of it,
        # 2^-25 = 2^-39 of the largest; times the keys' sum of magnitudes, in the exponent
        es = es + 2.0 ** -39 * q[:, h].abs().amax(1, keepdim=True) * kk.abs().sum(1).max() / d ** 0.5
        # weights rounded to f16 (half a step; the open page's to two bf16 terms, 2^-16), sums of their
        # products in fp32; a row's two sums (numerator, denominator) both carry the scores' error;
        # then one bf16 rounding
        av = p @ vv.abs()
        # what a 16-bit weight cannot hold: weights of full pages enter as f16 of at most 2^15 (the
        # largest is over 2^13: a row's maximum is rounded up to an integer, a step to a power of two),
        # so half a subnormal step, 2^-25, is at most 2^-38 of the largest weight times step; times a
        # code of at most 127, and 127 steps are a page's largest value
        small = len(kk) * 2.0 ** -38 * vv.abs().max()
        tol[:, h] = (av * (F11 + 2 * es + 2 * len(kk) * F24) * 1.01 + out[:, h].abs() * BF8 * 1.01 + small
                     + 1e-30)
        lse[h] = torch.logsumexp(s, 1) * 1.4426950408889634
    return out, tol, lse
