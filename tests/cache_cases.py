"""Paged caches made for the tests of the attention over them, the definition
of that attention in 64 bits, and the error that its arithmetic may have."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def make(seed, dtype, heads, kv_heads, dim, page, before, new, window=0, sinks=0, order="head", offsets=True,
         poison=True, spread=1.0):
    """A cache of sequences with ``before`` tokens and ``new`` ones, the pages
    in random order.  Whatever no query sees holds NaN when ``poison``."""
    g = torch.Generator().manual_seed(seed)
    dt = DTYPES[dtype]
    before, new = np.asarray(before, np.int64), np.asarray(new, np.int64)
    B, length = len(before), before + new
    have = -(-length // page)
    pool, width = int(have.sum()) + 3, max(int(have.max(initial=0)), 1) + 1
    table = torch.full((B, width), -1, dtype=torch.int32)
    place = torch.randperm(pool, generator=g).to(torch.int32)
    at = 0
    shape = (pool, kv_heads, page, dim)
    k = torch.full(shape, math.nan if poison else 7.0, dtype=dt)
    v = k.clone()
    rand = lambda *s: torch.randn(*s, generator=g).mul_(spread).to(dt)
    dense = []
    for b in range(B):
        table[b, :have[b]] = place[at:at + have[b]]
        at += int(have[b])
        L, n = int(length[b]), int(new[b])
        kb, vb = rand(L, kv_heads, dim), rand(L, kv_heads, dim)
        dense.append((kb, vb))
        t = torch.arange(L)
        if window and poison:
            t = t[(t > int(before[b]) - window) | (t < sinks)]
        if n == 0 and poison:
            t = t[:0]
        p, r = table[b].long()[t // page], t % page
        k[p, :, r], v[p, :, r] = kb[t], vb[t]
    T = int(new.sum())
    qkv = rand(T, heads + 2 * kv_heads, dim)      # a strided view, as a layer's fused product gives it
    if order == "token":
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)])) if offsets else None
    dev = lambda x: None if x is None else (x.transpose(1, 2).cuda().transpose(1, 2) if x.dim() == 4 else x.cuda())
    return dict(q=dev(qkv)[:, :heads], k=dev(k), v=dev(v), table=dev(table),
                length=torch.from_numpy(length.astype(np.int32)).cuda(), offset=dev(off), dense=dense,
                before=before, new=new, window=window, sinks=sinks, dtype=dtype, page=page)


def exact(c, scale=None, see=None):
    """(out, lse, bound on out's error, bound on lse's) in float64.  ``see(b, p, t)``
    replaces the visibility.

    The bound: the output's own rounding u |out|; each weight rounded to the
    16-bit type before the product with the values, u sum w |v| (and, in half
    precision, 2^-24 absolute for weights below its normal range, relative to a
    largest weight of 1); a score's error d = 2^-24 (dim + 4) sum |q| |k| scale,
    and 2^-22 |score| for scaling it and taking the exponential's argument,
    twice (weight and normaliser); sums over n tokens in fp32."""
    q = c["q"].double()
    T, H, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    half = c["dtype"] == "f16"
    u = 2.0 ** (-11 if half else -8)
    out = torch.zeros(T, H, D, dtype=torch.float64, device=q.device)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    first = 0
    for b, (a, n) in enumerate(zip(c["before"].tolist(), c["new"].tolist())):
        if n == 0:
            continue
        kb, vb = (x.to(q.device).double() for x in c["dense"][b])
        L = kb.shape[0]
        t = torch.arange(L, device=q.device)[None]
        p = torch.arange(a, a + n, device=q.device)[:, None]
        if see is not None:
            vis = see(b, p, t)
        else:
            vis = t <= p
            if c["window"]:
                vis = vis & ((t > p - c["window"]) | (t < c["sinks"]))
        for h in range(H):
            g = h // (H // kb.shape[1])
            rows = slice(first, first + n)
            s = (q[rows, h] @ kb[:, g].T.contiguous()) * scale
            s = torch.where(vis, s, -math.inf)
            m = s.amax(1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            w = torch.exp(s - m)
            l = w.sum(1, keepdim=True)
            some = l > 0
            l1 = torch.where(some, l, torch.ones_like(l))
            w = torch.where(vis, w / l1, torch.zeros_like(w))
            vv = torch.where(torch.isfinite(vb[:, g]), vb[:, g], torch.zeros_like(vb[:, g]))
            out[rows, h] = w @ vv
            lse[rows, h] = torch.where(some, m + torch.log(l1), torch.full_like(m, -math.inf))[:, 0]
            mag = (q[rows, h].abs() @ kb[:, g].abs().T.contiguous()) * scale
            mag = torch.where(vis, mag, torch.zeros_like(mag)).amax(1, keepdim=True)
            d = 2.0 ** -24 * (D + 4) * mag + 2.0 ** -22 * (mag + 4)
            av = w @ vv.abs()
            tol[rows, h] = u * out[rows, h].abs() + av * (1.01 * u + 2.02 * d + 2.0 ** -23 * L + 2.0 ** -20)
            if half:
                few = (vis.double() @ vv.abs()) / l1
                tol[rows, h] += 2.0 ** -24 * few + 2.0 ** -25
            tol_lse[rows, h] = (d + 2.0 ** -23 * L + 2.0 ** -20 + 2.0 ** -22 * lse[rows, h].abs().nan_to_num(0, 0, 0)[:, None])[:, 0]
        first += n
    return out, lse, tol, tol_lse


def check(c, got, lse, scale=None, see=None):
    out, ref_lse, tol, tol_lse = exact(c, scale, see)
    got = got.double()
    assert bool(torch.isfinite(got).all()), f"{int((~torch.isfinite(got)).sum())} values are not finite"
    off = (got - out).abs()
    worst = float((off / (tol + 1e-300)).max()) if off.numel() else 0.0
    assert bool((off <= tol).all()), f"{worst:.2f} times the bound, {int((off > tol).sum())} values"
    if lse is not None:
        lse = lse.double()
        none = torch.isinf(ref_lse)
        assert torch.equal(torch.isinf(lse) & (lse < 0), none)
        d = torch.where(none, torch.zeros_like(lse), lse - torch.where(none, torch.zeros_like(lse), ref_lse)).abs()
        d = torch.where(none, torch.zeros_like(d), d)
        assert bool((d <= tol_lse).all()), f"lse off by {float(d.max()):.3g}"
    return worst
