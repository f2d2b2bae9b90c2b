"""Plain references of the dense operators, in 64 bits, with the bounds that the operators' own rounding allows.

Dropout's generator is written here with numpy's 64-bit integers. The bounds are elementwise and follow
from the operations: a sum of n products in fp32 is off by at most (n + 8) 2^-24 of the sum of their
magnitudes in any order, an activation by its slope times that plus a few units of the 24th bit, and a result
stored in a 16-bit type by half its last bit.
"""
import math

import numpy as np
import torch

# half the last bit, relative: 2^-(fraction bits + 1)
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the spacing of the subnormal numbers
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


def philox(counter, key, rounds=7):
    """Philox4x32 of arrays of counters [.., 4] (uint64 holding 32 bits), key two 32-bit numbers."""
    M = np.uint64(0xFFFFFFFF)
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ k[0], q & M, (p >> np.uint64(32)) ^ c[3] ^ k[1], p & M]
        k = [(k[0] + np.uint64(0x9E3779B9)) & M, (k[1] + np.uint64(0xBB67AE85)) & M]
    return np.stack(c, axis=-1)


def kept(rows, F, p, seed, offset, first_row=0, first_group=0):
    """The mask of dropout at rows first_row.. and columns 4 * first_group..: a bool array [rows, F]."""
    groups = -(-F // 4)
    ctr = np.zeros((rows, groups, 4), dtype=np.uint64)
    ctr[..., 0] = np.arange(first_group, first_group + groups, dtype=np.uint64)
    ctr[..., 1] = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    ctr[..., 2], ctr[..., 3] = offset & 0xFFFFFFFF, offset >> 32
    words = philox(ctr, (seed & 0xFFFFFFFF, seed >> 32)).reshape(rows, groups * 4)[:, :F]
    return words >= np.uint64(round(p * 2 ** 32))


def act64(name, g):
    """(act(g), act'(g)) in 64 bits, and bounds on |act'| and |act''|."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), 1.1, 0.5
    if name == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi), 1.13, 0.8
    if name == "relu":
        return g.clamp_min(0), (g > 0).double(), 1.0, 0.0
    if name == "sigmoid":
        s = torch.sigmoid(g)
        return s, s * (1 - s), 0.25, 0.1
    return g, torch.ones_like(g), 1.0, 0.0


def gated64(x, wg, wu, bg, bu, act, mask=None, grad=None):
    """The block (and with `grad` its gradients) of the given tensors in 64 bits: a list of (value, bound),
    the bound without the output's own rounding. mask: kept / (1 - p) or None."""
    kind, K, N = x.dtype, x.shape[1], wg.shape[0]
    x, wg, wu = x.double(), wg.double(), wu.double()
    zero = torch.zeros(N, dtype=torch.float64, device=x.device)
    bg = zero if bg is None else bg.double()
    bu = zero if bu is None else bu.double()
    g, u = x @ wg.t() + bg, x @ wu.t() + bu
    eg = (K + 8) * U * (x.abs() @ wg.abs().t() + bg.abs())
    eu = (K + 8) * U * (x.abs() @ wu.abs().t() + bu.abs())
    a, da, l1, l2 = act64(act, g)
    m = torch.ones_like(g) if mask is None else mask.double()
    # the activation itself: a few units, and the short exponential's error grows with its argument
    ea = l1 * eg + 32 * U * (1 + g.abs()) * (a.abs() + g.abs() * 2.0 ** -20 + 2.0 ** -100)
    eda = l2 * eg + 32 * U * (1 + g.abs()) * (1 + g.abs())
    if act == "relu":
        eda = (g.abs() <= eg).double() + 0 * eda   # the step is exact away from 0
    out = m * a * u
    res = [(out, m * (ea * u.abs() + a.abs() * eu + ea * eu) + 4 * U * out.abs())]
    if grad is None:
        return res
    d = m * grad.double()
    dg, du = d * u * da, d * a
    r = EPS[kind] if kind != torch.float32 else U
    edg = d.abs() * (eda * u.abs() + da.abs() * eu + eda * eu) + 4 * U * dg.abs()
    edu = d.abs() * ea + 4 * U * du.abs()
    rg, ru = edg + r * (dg.abs() + edg) + TINY[kind], edu + r * (du.abs() + edu) + TINY[kind]
    M = x.shape[0]
    res.append((dg @ wg + du @ wu, rg @ wg.abs() + ru @ wu.abs() +
                (2 * N + 8) * U * ((dg.abs() + rg) @ wg.abs() + (du.abs() + ru) @ wu.abs())))
    for t, e in ((dg, rg), (du, ru)):
        res.append((t.t() @ x, e.t() @ x.abs() + (M + 8) * U * ((t.abs() + e).t() @ x.abs())))
    for t, e in ((dg, edg), (du, edu)):
        res.append((t.sum(0), e.sum(0) + (M + 8) * U * (t.abs() + e).sum(0)))
    return res


def check(got, ref, bound, what=""):
    """|got - ref| within bound and got's own last bit."""
    assert got.shape == ref.shape, f"{what}: shape {tuple(got.shape)}, expected {tuple(ref.shape)}"
    lim = bound + EPS[got.dtype] * (ref.abs() + bound) + TINY[got.dtype]
    err = (got.double() - ref).abs()
    bad = ~(err <= lim)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {i}: {float(got[i])!r}, "
                             f"expected {float(ref[i])!r}, error {float(err[i]):.3e} > {float(lim[i]):.3e}")
