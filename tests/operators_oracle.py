"""The layer operators (LayerNorm, dropout, differential attention) in 64 bits on
the CPU, from their formulas, and bounds on what the kernels' roundings cost.

A value stored in a type is off by at most half a step, HALF[dtype] relative to
it.  Inside, the bf16 kernels round the operands of the second products
(probabilities, gradients of the scores) to bf16 once; everything else is fp32,
whose sums of n terms are bounded by n 2^-24 times the sum of magnitudes."""
import math

import numpy as np
import torch

EPS32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def layer_norm(x, w, b, eps, dy=None):
    """(y, its bound), and with dy also dx, dw, db with their bounds."""
    half = HALF[x.dtype]
    x64 = x.double().reshape(-1, x.shape[-1])
    C = x64.shape[1]
    w64 = torch.ones(C, dtype=torch.float64) if w is None else w.double()
    b64 = torch.zeros(C, dtype=torch.float64) if b is None else b.double()
    mean = x64.mean(-1, keepdim=True)
    xc = x64 - mean
    rstd = 1.0 / torch.sqrt((xc * xc).mean(-1, keepdim=True) + eps)
    xh = xc * rstd
    y = xh * w64 + b64
    # A lane adds up to 16 values and the row up to 8 + 2 partial sums: 32 roundings
    # of the mean's terms, as many for the variance, and a handful after that.
    mag = (x64.abs().max(-1, keepdim=True).values + mean.abs()) * rstd
    e_xh = 80 * EPS32 * (mag + xh.abs()) + 80 * EPS32 * mag * xh.abs()
    out = [(y, half * y.abs() + e_xh * w64.abs() + 4 * EPS32 * (y.abs() + b64.abs()))]
    if dy is not None:
        g0 = dy.double().reshape(-1, C)
        g = g0 * w64
        m0, m1 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
        dx = rstd * (g - m0 - xh * m1)
        ag, agx = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True)
        e = rstd * (80 * EPS32 * (g.abs() + ag + xh.abs() * agx) + e_xh * agx +
                    xh.abs() * (g.abs() * e_xh).mean(-1, keepdim=True))
        rows = x64.shape[0]
        # A lane adds the rows of its workgroup, then up to 1024 workgroups are joined.
        n = min(rows, rows / 1024 + 64) + 64
        dw, db = (g0 * xh).sum(0), g0.sum(0)
        out += [(dx, half * dx.abs() + e),
                (dw, half * dw.abs() + n * EPS32 * (g0 * xh).abs().sum(0) +
                 (g0.abs() * e_xh).sum(0)),
                (db, half * db.abs() + n * EPS32 * g0.abs().sum(0))]
    shape = x.shape
    return [(v.reshape(shape), e.reshape(shape)) if v.numel() == x.numel() and v.dim() == 2
            else (v, e) for v, e in out]


def keep_mask(n, p, seed, offset):
    """Elements that dropout keeps: Philox-4x32-10, word by word in Python integers."""
    T = math.floor(p * 65536 + 0.5)
    out = np.zeros(n, dtype=bool)
    for blk in range((n + 7) // 8):
        c = [blk & 0xFFFFFFFF, blk >> 32, offset & 0xFFFFFFFF, offset >> 32]
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        for j in range(min(8, n - 8 * blk)):
            out[8 * blk + j] = ((c[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= T
    return torch.from_numpy(out)


def visible(W, nq, nk, causal, kv_len):
    """bool [W, nq, nk]"""
    i, j = torch.arange(nq)[:, None], torch.arange(nk)[None, :]
    out = torch.zeros(W, nq, nk, dtype=torch.bool)
    for w in range(W):
        n = nk if kv_len is None else min(max(int(kv_len[w]), 0), nk)
        out[w] = (j < n) & {0: j >= 0, 1: j <= i, 2: j <= n - nq + i}[causal]
    return out


def diff_attention(q, k, v, lam, causal=0, kv_len=None, scale=None, do=None, short=256):
    """[(value, bound)] of O, and with do of dq, dk, dv, dlam.  Masked keys and values
    are left out, not multiplied by zero."""
    dt = q.dtype
    half, low = HALF[dt], (2.0 ** -8 if dt == torch.bfloat16 else 0.0)
    W, H2, nq, d = q.shape
    H, G, nk, dv = H2 // 2, v.shape[1], v.shape[2], v.shape[3]
    R = H // G
    s = 1.0 / math.sqrt(d) if scale is None else scale
    see = visible(W, nq, nk, causal, kv_len)
    used = see.any(1)[:, None, :, None]                       # keys that some query sees
    q64 = q.double()
    k64 = torch.where(used, k.double(), 0.0)
    v64 = torch.where(used, v.double(), 0.0)
    # [W, G, 1, R nq, .] queries against the keys of their group
    def grouped(x):
        return x.reshape(W, G, R * nq, x.shape[-1])
    vis = see[:, None, None].expand(W, G, R, nq, nk).reshape(W, G, R * nq, nk)
    qs = q64.reshape(W, G, R, 2, nq, d)
    P, mags = [], []
    for a in range(2):
        qa, ka = grouped(qs[:, :, :, a]), k64.reshape(W, G, 2, nk, d)[:, :, a]
        S = qa @ ka.transpose(-1, -2) * s
        S = S.masked_fill(~vis, -math.inf)
        m = S.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        e = torch.exp(S - m)
        t = e.sum(-1, keepdim=True)
        P.append(e / torch.where(t == 0, 1.0, t))
        mags.append((qa.abs() @ ka.abs().transpose(-1, -2)).amax() * s if S.numel() else 0.0)
    l = lam.double().reshape(1, G, R, 1, 1).expand(W, G, R, nq, 1).reshape(W, G, R * nq, 1)
    # Relative error of a probability: its score's, the row sum's over nk terms (each lane
    # adds at most half of them, in tiles), exp2 and logarithm.
    eP = EPS32 * ((d + 16) * max(mags) * 2 + 64 + nk / 16)
    A = P[0] + l.abs() * P[1]
    a = P[0] - l * P[1]
    O, AV = a @ v64, A @ v64.abs()
    eAcc = EPS32 * (nk / 4 + 64)
    eO = (low + eP + eAcc) * AV
    o = O.reshape(W, H, nq, dv)
    out = [(o, half * o.abs() + eO.reshape(o.shape) * (1 + half))]
    if do is None:
        return out
    g = grouped(do.double())
    X = g @ v64.transpose(-1, -2)
    aX = g.abs() @ v64.abs().transpose(-1, -2)
    eX = EPS32 * (dv + 8) * aX
    D = [(p * X).sum(-1, keepdim=True) for p in P]
    if nk > short:
        # dO . O_a from the fp32 outputs: off by their products' operands and their sums
        dot = EPS32 * (dv + 8)
        eD = [(g.abs() * ((low + eP + eAcc) * (p @ v64.abs()) + dot * (p @ v64).abs()))
              .sum(-1, keepdim=True) for p in P]
        if dt == torch.float32:      # D_1 from O and D_2
            eD[0] = ((g.abs() * (eO + (dot + half) * O.abs())).sum(-1, keepdim=True) +
                     l.abs() * eD[1])
    else:
        eD = [(p * (eX + (eP + EPS32 * (nk + 8)) * X.abs())).sum(-1, keepdim=True) for p in P]
    w = [1.0, -l]
    dS = [w[i] * P[i] * (X - D[i]) for i in range(2)]
    eS = [(l.abs() if i else 1.0) * P[i] * (eD[i] + eX + (eP + 4 * EPS32) * (X - D[i]).abs()) +
          low * dS[i].abs() * (1 + eP) for i in range(2)]
    eS = [e + low * e for e in eS]
    gq = torch.zeros(W, G, R, 2, nq, d, dtype=torch.float64)
    bq = torch.zeros_like(gq)
    gk = torch.zeros(W, G, 2, nk, d, dtype=torch.float64)
    bk = torch.zeros_like(gk)
    rows = R * nq
    for i in range(2):
        qa, ka = grouped(qs[:, :, :, i]), k64.reshape(W, G, 2, nk, d)[:, :, i]
        x, e = s * (dS[i] @ ka), s * ((eS[i] + eAcc * dS[i].abs()) @ ka.abs())
        gq[:, :, :, i] = x.reshape(W, G, R, nq, d)
        bq[:, :, :, i] = (e + half * x.abs() + half * e).reshape(W, G, R, nq, d)
        x = s * (dS[i].transpose(-1, -2) @ qa)
        e = s * ((eS[i] + EPS32 * (rows / 4 + 64) * dS[i].abs()).transpose(-1, -2) @ qa.abs())
        gk[:, :, i], bk[:, :, i] = x, e + half * x.abs() + half * e
    gv = a.transpose(-1, -2) @ g
    ev = ((low * a.abs() + (1 + low) * eP * A + EPS32 * (rows / 4 + 64) * a.abs())
          .transpose(-1, -2) @ g.abs())
    rowlam = D[1].reshape(W, H, nq)
    erow = (P[1] * (eX + (eP + EPS32 * (nk + 8)) * X.abs())).sum(-1).reshape(W, H, nq)
    gl = -rowlam.sum((0, 2))
    el = erow.sum((0, 2)) + EPS32 * (W * nq / 512 + 64) * rowlam.abs().sum((0, 2))
    return out + [(gq.reshape(q.shape), bq.reshape(q.shape)),
                  (gk.reshape(k.shape), bk.reshape(k.shape)),
                  (gv, ev + half * gv.abs() + half * ev), (gl, el)]


def check(got, pair, what):
    ref, bound = pair
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    x = got.detach().double().cpu()
    assert torch.isfinite(x).all(), f"{what}: not finite"
    off = (x - ref).abs()
    over = off - bound
    worst = float((off / bound.clamp_min(1e-300)).max()) if off.numel() else 0.0
    print(f"{what}: error {worst:.2f} of its bound, rms {float(off.square().mean().sqrt()) if off.numel() else 0:.2e}")
    assert not (over > 1e-37).any(), f"{what}: {worst:.2f} of the bound"
