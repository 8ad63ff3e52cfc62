"""64-bit forms of the operators around the MoE layer, and how far roundings may take a result from them."""
import math

import torch

HALF_BF16 = 2.0 ** -8          # a rounding to bf16 moves a value by at most this share of it
HALF_E4M3 = 2.0 ** -4          # the same of e4m3, for values from 2^-6 on; below, by at most 2^-10
E4M3 = torch.float8_e4m3fn
FLOOR = 2.0 ** -100


def groups(y):
    """[T, d] -> [T, groups, 128], filled up with zeros."""
    T, d = y.shape
    G = -(-d // 128)
    return torch.nn.functional.pad(y, (0, G * 128 - d)).reshape(T, G, 128)


def scales_of(y):
    """[groups, T]"""
    return (groups(y).abs().amax(2).clamp_min(FLOOR) / 448.0).t()


def spread(scale, d):
    """[groups, T] -> [T, d]"""
    return scale.t().repeat_interleave(128, 1)[:, :d]


def near(got, want, tol, what=""):
    got, want = got.double().cpu(), want.double().cpu()
    tol = torch.as_tensor(tol, dtype=torch.float64).cpu().expand_as(want)
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}: got {got[bad][0]:.9g}, " \
                                f"want {want[bad][0]:.9g} +- {tol[bad][0]:.3g}"


def attention(q, k, v, lengths, scale, window=0, left_out=None):
    """q [T, H, D], k and v [T, L, Hk, D] (what each token's row of the table leads to) in 64 bits.  Returns out, lse, and the bound on out
    and lse: each probability is rounded to bf16, the scores carry the error of an fp32 sum of D products."""
    T, H, D = q.shape
    group = H // k.shape[2]
    out, tol = torch.zeros((2, T, H, D), dtype=torch.float64)
    lse, tol_lse = torch.full((T, H), -math.inf, dtype=torch.float64), torch.zeros((T, H), dtype=torch.float64)
    for t in range(T):
        n = min(max(int(lengths[t]), 0), k.shape[1])
        at = torch.arange(max(n - window, 0) if window else 0, n)
        if left_out is not None:
            at = at[~left_out[t, at]]
        if len(at) == 0:
            continue
        kt, vt = (x[t, at].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))       # [H, positions, D]
        s = (kt @ q[t][:, :, None])[..., 0] * scale
        size = (kt.abs() @ q[t].abs()[:, :, None])[..., 0] * abs(scale)
        lse[t] = torch.logsumexp(s, 1)
        p = torch.softmax(s, 1)[:, None]
        out[t] = (p @ vt)[:, 0]
        near_v = (p @ vt.abs())[:, 0]
        # the hardware's exponential and the fp32 sums besides
        ds = (D + 8) * 2.0 ** -24 * size.amax(1) + 2e-6 + len(at) * 2.0 ** -24 / 8
        tol[t] = HALF_BF16 * (out[t].abs() + near_v) + 2 * ds[:, None] * near_v + 1e-30
        tol_lse[t] = ds + 1e-6 * lse[t].abs()
    return out, lse, tol, tol_lse
