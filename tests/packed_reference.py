"""The packed cache's format and the attention over it, written out in 64 bits (numpy and torch on the CPU)."""
import math

import numpy as np
import torch

GROUP = 32


def quantise(x):
    """x (..., d) -> (codes int (..., d/32, 32), scales float64 holding fp16 values (..., d/32))."""
    x = np.asarray(x.double().cpu() if torch.is_tensor(x) else x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    finite = np.isfinite(g).all(-1)
    safe = np.where(finite[..., None], g, 0.0)
    peak = np.take_along_axis(safe, np.abs(safe).argmax(-1)[..., None], -1)[..., 0]   # argmax: the first of equals
    with np.errstate(over="ignore"):
        s = np.clip(peak / -8.0, -65504.0, 65504.0).astype(np.float16).astype(np.float64)
    code = np.where(s[..., None] == 0, 0.0, np.clip(np.rint(safe / np.where(s == 0, 1.0, s)[..., None]), -8, 7))
    return code.astype(np.int64), np.where(finite, s, np.nan)


def values(code, s):
    v = code * s[..., None]
    return torch.from_numpy(v.reshape(*v.shape[:-2], v.shape[-2] * GROUP))


def packed_values(x):
    """What rows x (..., d) read back as, float64."""
    return values(*quantise(x))


def attend(q, k, v, lens, first, scale, dtype, blocks=False):
    """q (b, I, Hq, d), k / v (b, n, Hkv, d) float64 -> out, and per output element the sum of p |v| and the largest relative
    error that the sums of the logits may put on a weight.  blocks: keys and values may go through fp16 (calls of many queries)."""
    b, I, Hq, d = q.shape
    n, Hkv = k.shape[1], k.shape[2]
    out = torch.zeros(b, I, Hq, d, dtype=torch.float64)
    spread = torch.zeros_like(out)
    slack = torch.zeros(b, I, Hq, 1, dtype=torch.float64)
    for s in range(b):
        lo, len_ = max(first[s], 0), min(max(lens[s], 0), n)
        if len_ <= lo:
            continue
        seen = torch.arange(lo, len_) < (len_ - (I - 1 - torch.arange(I)))[:, None]      # (I, rows)
        some = seen.any(1, keepdim=True)
        for h in range(Hq):
            kk, vv = k[s, lo:len_, h // (Hq // Hkv)], v[s, lo:len_, h // (Hq // Hkv)]
            qq = q[s, :, h]
            logit = qq @ kk.T * scale
            p = torch.where(some, torch.softmax(torch.where(seen | ~some, logit, -math.inf), 1), 0.0)
            out[s, :, h] = p @ vv
            spread[s, :, h] = p @ vv.abs()
            if dtype == torch.bfloat16:
                # A group's sum runs over 32 products u q (u <= 15) from -8 sum q: at most 40 additions of at most 23 sum |q|,
                # each off by a step of fp32, 2^-23; times the scale, an eighth of the group's largest |k| (1 + 2^-10).
                size = kk.abs().view(len(kk), -1, GROUP).amax(-1) / 8 * (1 + 2 ** -10)
                err = qq.abs().view(I, -1, GROUP).sum(-1) @ size.T * (23 * 40 * 2.0 ** -23)
                # up to four query rows of a cache are integers, each element off by half a step, 2^-15 of the row's largest
                if I * (Hq // Hkv) <= 4:
                    err = err + kk.abs().sum(-1) * qq.abs().amax(-1, keepdim=True) * 2.0 ** -14
                if blocks:   # every key may be off by half a step of fp16, and d products are added
                    err = torch.maximum(err, qq.abs() @ kk.abs().T * (2.0 ** -11 + d * 2.0 ** -23))
            else:
                # 64 products (two halves of q, which leave 2^-22 of it out) from 0, then the groups
                err = qq.abs() @ kk.abs().T * (72 * 2.0 ** -23 + 2.0 ** -22)
            err = err * scale + logit.abs() * 8 * 2.0 ** -23
            slack[s, :, h] = 2 * torch.where(seen, err, 0.0).amax(1, keepdim=True)
    return out, spread, slack


def bound(out, spread, slack, dtype, n, vmax, blocks=False):
    """How far an output may be off.  n rows, |value| <= vmax."""
    steps = n / 4 + 100              # additions into one element: a quarter of the rows a warp, the warps, the splits, the division
    if dtype == torch.bfloat16:
        weight = 2 * 2.0 ** -11      # p to fp16, p * s to fp16 (blocks: the value to fp16)
        last = 2.0 ** -8             # the output
        # sums of w u (u <= 15) and of 8 w: at most spread + 2 * 8 * s, s <= vmax / 8
        sums = steps * 2.0 ** -23 * (spread + 2 * vmax)
        if blocks:                   # the values themselves, one sum over all rows
            sums = sums + n * 2.0 ** -23 * spread
    else:
        weight = 2 * 2.0 ** -21      # two fp16 numbers each
        last = 2.0 ** -24
        sums = steps * 2.0 ** -23 * spread
    weight = weight + 2.0 ** -21 + slack            # 2^-21: ex2
    tiny = n * 2.0 ** -33 * vmax                    # fp16 weights below 2^-14 of 2^12
    return last * out.abs() + weight * spread + sums + tiny + 1e-30
