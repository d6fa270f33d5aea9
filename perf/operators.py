"""Operators for training and serving window-attention layers, with their plain
forms: layer normalisation, dropout from a counter-based generator, and
differential attention.

Kinds of case
  norm       LayerNorm over the channels of a list of tokens
  norm_grad  its forward and backward pass: output and the gradients of the
             input, the weight and the bias
  drop       dropout of a branch added to the residual stream
  drop_grad  that, and the gradient of the branch
  attn       differential attention, O = (softmax(s Q1 K1^T) - lam softmax(s Q2 K2^T)) V
  attn_grad  its forward and backward pass: O and the gradients of Q, K, V and lam

Where `own` is true, `run` calls the framework; otherwise it evaluates the
formulas with elementary torch operations in fp32.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _norm(name, kind, rows, C, dtype):
    return dict(name=name, kind=kind, rows=rows, C=C, dtype=dtype)


def _drop(name, kind, n, p, dtype):
    return dict(name=name, kind=kind, n=n, p=p, dtype=dtype)


def _attn(name, kind, windows, heads, kv_heads, n_q, n_k, d, dv, dtype, causal="none",
          ragged=False, layout="heads"):
    return dict(name=name, kind=kind, windows=windows, heads=heads, kv_heads=kv_heads, n_q=n_q,
                n_k=n_k, d=d, dv=dv, dtype=dtype, causal=causal, ragged=ragged, layout=layout)


def listed():
    return [
        # One 8 x 8 window of a SwinIR layer (180 channels): the smallest call.
        _norm("norm_window_bf16", "norm", 64, 180, "bf16"),
        # A training step's norm of that layer on four 128 x 128 crops.
        _norm("norm_crops_bf16", "norm_grad", 4 * 128 * 128, 180, "bf16"),
        # A wide layer with an odd channel count and a ragged token count, fp32.
        _norm("norm_wide_odd_f32", "norm_grad", 20011, 1021, "f32"),
        # Dropout behind the attention of one window: latency.
        _drop("drop_window_bf16", "drop", 64 * 180, 0.1, "bf16"),
        # The residual branch of a SwinIR layer in a training step, both directions.
        _drop("drop_crops_bf16", "drop_grad", 4 * 128 * 128 * 180, 0.1, "bf16"),
        # A large fp32 activation whose size no vector width divides.
        _drop("drop_large_odd_f32", "drop", 50000003, 0.25, "f32"),
        # A SwinIR layer's windows on a 256 x 256 map: six heads of width 30, read
        # from the projection's output as it lies.
        _attn("attn_8x8_bf16", "attn", 1024, 6, 6, 64, 64, 30, 60, "bf16", layout="tokens"),
        # Fine-tuning with enlarged 16 x 16 windows.
        _attn("attn_16x16_grad_bf16", "attn_grad", 256, 6, 6, 256, 256, 32, 64, "bf16",
              layout="tokens"),
        # Global attention over 64 x 64 maps, both directions: the largest case.
        _attn("attn_global_grad_bf16", "attn_grad", 2, 8, 8, 4096, 4096, 64, 128, "bf16"),
        # A padded batch of sequences of different lengths (one is empty), causal,
        # shared key and value heads, widths that no tile divides, fp32.
        _attn("attn_ragged_grad_f32", "attn_grad", 5, 8, 2, 777, 777, 44, 88, "f32",
              causal="start", ragged=True),
        # A new token for each of 16 sequences over a cache of up to 8192.
        _attn("attn_token_bf16", "attn", 16, 16, 4, 1, 8192, 64, 128, "bf16", causal="end",
              ragged=True),
        # The smallest attention call: one token, one short cache, fp32.
        _attn("attn_token_small_f32", "attn", 1, 6, 6, 1, 197, 30, 60, "f32", causal="end"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = None


def _draw(rng):
    kind = rng.choice(["norm", "norm_grad", "drop", "drop_grad", "attn", "attn", "attn_grad",
                       "attn_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if kind.startswith("norm"):
        # At two channels the input's gradient is rounding alone: it starts at four.
        C = rng.choice([rng.randint(4, 64), _log_int(rng, 16, 4096), 4 * rng.randint(8, 256)])
        c = _norm("", kind, _log_int(rng, 1, 200000), C, dtype)
    elif kind.startswith("drop"):
        c = _drop("", kind, _log_int(rng, 1, 50000000), rng.choice([0.0, 0.05, 0.1, 0.5, 0.9]), dtype)
    else:
        d = rng.choice([rng.randint(1, 64), rng.choice([16, 30, 32, 48, 64])])
        dv = rng.choice([2 * d, 2 * d, rng.randint(1, 128)])
        kv = rng.choice([1, 2, 4, 6])
        heads = kv * rng.choice([1, 1, 2, 4])
        form = rng.choice(["window", "padded", "token"])
        n_k = _log_int(rng, 1, 4096)
        n_q, causal, ragged = n_k, rng.choice(["none", "start"]), False
        if form == "padded":
            ragged = True
        elif form == "token":
            n_q, n_k, causal, ragged = rng.randint(1, 8), _log_int(rng, 8, 8192), "end", True
        c = _attn("", kind, _log_int(rng, 1, 1024), heads, kv, n_q, n_k, d, dv, dtype, causal,
                  ragged, rng.choice(["heads", "tokens"]))
    del c["name"]
    return c


def draw(rng):
    """A case of the same ranges that costs no more than the largest listed one."""
    global _MOST
    if _MOST is None:
        all_work = [work(c) for c in listed()]
        _MOST = {k: max(w[k] for w in all_work) for k in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        w = work(c)
        # The plain form's maps: at most what the largest listed case has.
        maps = 2 * c["windows"] * c["heads"] * c["n_q"] * c["n_k"] if "heads" in c else 0
        if all(w[k] <= _MOST[k] for k in _MOST) and maps <= 1 << 29:
            return c


def _lengths(case):
    """Keys of each window: all of them, or a ragged batch with an empty one."""
    W, n = case["windows"], case["n_k"]
    if not case["ragged"]:
        return [n] * W
    return [0 if W > 2 and w == W // 2 else max(1, n - (w * 7919) % max(1, (2 * n) // 3))
            for w in range(W)]


def _pairs(case):
    """Visible (query, key) pairs of one head, over all windows."""
    total = 0
    for ln in _lengths(case):
        nq = case["n_q"]
        if case["causal"] == "none":
            total += nq * ln
        else:
            first = 0 if case["causal"] == "start" else ln - nq
            # sum over i of clamp(first + i + 1, 0, ln)
            lo = max(0, -first)                        # first row that sees a key
            hi = min(nq, max(lo, ln - first))          # rows below hi see fewer than ln keys
            k = hi - lo
            total += k * (first + lo + 1) + k * (k - 1) // 2 + (nq - hi) * ln
    return total


def work(case):
    """What one pass cannot do without: every input read once, every output
    written once, and the products of the formulas."""
    e = _BYTES[case["dtype"]]
    kind = case["kind"]
    if kind.startswith("norm"):
        n, C = case["rows"] * case["C"], case["C"]
        # x and y; with gradients also dy and dx, the weights and their gradients
        if kind == "norm":
            return {"bytes": (2 * n + 2 * C) * e, "flops": 8 * n}
        return {"bytes": (4 * n + 4 * C) * e, "flops": 22 * n}
    if kind.startswith("drop"):
        n = case["n"]
        # x, residual and sum; with gradients also dy and dx
        return {"bytes": (5 if kind == "drop_grad" else 3) * n * e, "flops": 2 * n}
    W, H, G, d, dv = (case[k] for k in ("windows", "heads", "kv_heads", "d", "dv"))
    q, o = W * H * case["n_q"] * 2 * d, W * H * case["n_q"] * dv
    kv = G * sum(_lengths(case)) * (2 * d + dv)
    pairs = H * _pairs(case)
    if kind == "attn":
        return {"bytes": (q + o + kv) * e + 4 * H, "flops": pairs * (4 * d + 2 * dv)}
    return {"bytes": (2 * q + 2 * o + 2 * kv) * e + 8 * H,
            "flops": pairs * (12 * d + 6 * dv)}


# ---- inputs -------------------------------------------------------------------


def _tokens(x):
    """[windows][heads][tokens][width] values laid out token by token, as the
    output of a projection holds them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    kind = case["kind"]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dt)

    s = dict(case)
    if kind.startswith("norm"):
        rows, C = case["rows"], case["C"]
        x = torch.randn(rows, C, generator=g, device="cuda")
        # tokens of an activation: each with a mean and a scale of its own
        x = x * (0.5 + torch.rand(rows, 1, generator=g, device="cuda"))
        s["x"] = (x + torch.randn(rows, 1, generator=g, device="cuda")).to(dt)
        s["w"], s["b"] = normal(C, std=0.2, mean=1.0), normal(C, std=0.2)
        s["dy"] = normal(rows, C) if kind == "norm_grad" else None
    elif kind.startswith("drop"):
        n = case["n"]
        s["x"], s["res"] = normal(n), normal(n)
        s["dy"] = normal(n) if kind == "drop_grad" else None
        s["seed"], s["offset"] = 0x9D2C5680 + 0x1234567 * seed, 3 + seed
    else:
        W, H, G, nq, nk, d, dv = (case[k] for k in ("windows", "heads", "kv_heads", "n_q", "n_k",
                                                     "d", "dv"))
        lay = _tokens if case["layout"] == "tokens" else (lambda x: x)
        s["q"] = lay(normal(W, 2 * H, nq, d))
        s["k"] = lay(normal(W, 2 * G, nk, d))
        s["v"] = lay(normal(W, G, nk, dv, mean=0.25))
        s["lam"] = 0.2 + 0.6 * torch.rand(H, generator=g, device="cuda")
        s["do"] = lay(normal(W, H, nq, dv)) if kind == "attn_grad" else None
        s["kv_len"] = (torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
                       if case["ragged"] else None)
    return s


# ---- the plain forms ----------------------------------------------------------


def _plain_norm(s):
    dt = s["x"].dtype
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(-1, keepdim=True) + 1e-5)
    xh = xc * rstd
    y = (xh * w + b).to(dt)
    if s["kind"] == "norm":
        return y
    dy = s["dy"].float()
    gw = dy * w
    dx = rstd * (gw - gw.mean(-1, keepdim=True) - xh * (gw * xh).mean(-1, keepdim=True))
    return y, dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)


def _mul32(a, m):
    """High and low 32 bits of a * m (values below 2^32 in int64)."""
    prod = a * m                       # wraps modulo 2^64: the bits are right
    return (prod >> 32) & 0xFFFFFFFF, prod & 0xFFFFFFFF


def _keep(n, p, seed, offset, device):
    """Which of n elements stay: 16 bits per element from the Philox-4x32
    counter-based generator with 10 rounds, eight elements to a counter."""
    blocks = (n + 7) // 8
    i = torch.arange(blocks, dtype=torch.int64, device=device)
    c0, c1 = i & 0xFFFFFFFF, i >> 32
    c2, c3 = (torch.full_like(i, v) for v in (offset & 0xFFFFFFFF, (offset >> 32) & 0xFFFFFFFF))
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack((c0, c1, c2, c3), 1)
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[:n]
    return bits >= int(math.floor(p * 65536 + 0.5))


def _plain_drop(s):
    dt = s["x"].dtype
    T = int(math.floor(s["p"] * 65536 + 0.5))
    scale = 65536.0 / (65536 - T)
    keep = _keep(s["n"], s["p"], s["seed"], s["offset"], s["x"].device)
    y = (s["res"].float() + torch.where(keep, s["x"].float() * scale, 0.0)).to(dt)
    if s["kind"] == "drop":
        return y
    return y, torch.where(keep, s["dy"].float() * scale, 0.0).to(dt)


def _visible(s, device):
    """[windows][n_q][n_k]: which keys each query sees (None: all of them)."""
    if s["causal"] == "none" and s["kv_len"] is None:
        return None
    j = torch.arange(s["n_k"], device=device)
    i = torch.arange(s["n_q"], device=device)
    ln = (s["kv_len"].long() if s["kv_len"] is not None
          else torch.full((s["windows"],), s["n_k"], device=device))
    vis = (j < ln[:, None])[:, None, :]
    if s["causal"] == "start":
        vis = vis & (j[None, :] <= i[:, None])
    elif s["causal"] == "end":
        vis = vis & (j <= (i + ln[:, None] - s["n_q"])[:, :, None])
    return vis.expand(s["windows"], s["n_q"], s["n_k"])


def _plain_attn(s):
    W, H, G, nq, nk, d, dv = (s[k] for k in ("windows", "heads", "kv_heads", "n_q", "n_k", "d",
                                              "dv"))
    R, dt, scale = H // G, s["q"].dtype, 1.0 / math.sqrt(d)
    # Queries of the R heads that share keys, map by map: [W][G][2][R nq][d].
    q = s["q"].float().reshape(W, G, R, 2, nq, d).transpose(2, 3).reshape(W, G, 2, R * nq, d)
    k = s["k"].float().reshape(W, G, 2, nk, d)
    v = s["v"].float().contiguous()
    lam = s["lam"].reshape(1, G, R, 1, 1).expand(W, G, R, nq, 1).reshape(W, G, R * nq, 1)
    p = q @ k.transpose(-1, -2) * scale
    vis = _visible(s, q.device)
    if vis is not None:
        hidden = ~vis[:, None, None, None]
        p = p.reshape(W, G, 2, R, nq, nk).masked_fill_(hidden, -math.inf).reshape(p.shape)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = (p - m).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    p1, p2 = p[:, :, 0], p[:, :, 1]
    a = p1 - lam * p2
    o = (a @ v).reshape(W, H, nq, dv).to(dt)
    if s["kind"] == "attn":
        return o
    do = s["do"].float().reshape(W, G, R * nq, dv)
    g_v = (a.transpose(-1, -2) @ do).to(dt)
    del a
    x = do @ v.transpose(-1, -2)
    d1 = (p1 * x).sum(-1, keepdim=True)
    d2 = (p2 * x).sum(-1, keepdim=True)
    g_lam = -d2.reshape(W, H, nq).sum((0, 2))
    ds = torch.stack((p1 * (x - d1), -lam * (p2 * (x - d2))), 2) * scale
    g_q = (ds @ k).reshape(W, G, 2, R, nq, d).transpose(2, 3).reshape(W, 2 * H, nq, d).to(dt)
    g_k = (ds.transpose(-1, -2) @ q).reshape(W, 2 * G, nk, d).to(dt)
    return o, g_q, g_k, g_v, g_lam


# ---- the framework's calls ----------------------------------------------------


def _own_norm(s):
    from paper_2506_08520_amd import binding as B
    if s["kind"] == "norm":
        return B.nystra_layer_norm_forward(s["x"], s["w"], s["b"])
    y, mean, rstd = B.nystra_layer_norm_forward(s["x"], s["w"], s["b"], with_stats=True)
    return (y, *B.nystra_layer_norm_backward(s["dy"], s["x"], s["w"], mean, rstd))


def _own_drop(s):
    from paper_2506_08520_amd import binding as B
    y = B.nystra_dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["res"])
    if s["kind"] == "drop":
        return y
    return y, B.nystra_dropout(s["dy"], s["p"], s["seed"], s["offset"])


def _own_attn(s):
    from paper_2506_08520_amd import binding as B
    causal = {"none": B.CAUSAL_NONE, "start": B.CAUSAL_START, "end": B.CAUSAL_END}[s["causal"]]
    q, k, v, lam, kv_len = s["q"], s["k"], s["v"], s["lam"], s["kv_len"]
    if s["kind"] == "attn":
        return B.nystra_diff_attn_forward(q, k, v, lam, causal=causal, kv_len=kv_len)
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, causal=causal, kv_len=kv_len,
                                          with_saved=True)
    return (o, *B.nystra_diff_attn_backward(s["do"], q, k, v, lam, o, saved, causal=causal,
                                            kv_len=kv_len))


def run(state):
    kind = state["kind"].split("_")[0]
    if own:
        return {"norm": _own_norm, "drop": _own_drop, "attn": _own_attn}[kind](state)
    return {"norm": _plain_norm, "drop": _plain_drop, "attn": _plain_attn}[kind](state)


# ---- in 64 bits, from the definitions -----------------------------------------


def _exact_norm(s):
    x = s["x"].double().requires_grad_()
    w, b = s["w"].double().requires_grad_(), s["b"].double().requires_grad_()
    var = (x ** 2).mean(-1) - x.mean(-1) ** 2
    y = (x - x.mean(-1)[:, None]) / (var[:, None] + 1e-5).sqrt() * w + b
    if s["kind"] == "norm":
        return y.detach()
    return (y.detach(), *torch.autograd.grad(y, (x, w, b), s["dy"].double()))


def _exact_keep(n, p, seed, offset):
    """The generator's bits again, in numpy's unsigned 64-bit integers."""
    u, mask, half = np.uint64, np.uint64(0xFFFFFFFF), np.uint64(32)
    ctr = np.zeros((4, (n + 7) // 8), dtype=u)
    ctr[0] = np.arange((n + 7) // 8, dtype=u)
    ctr[1] = ctr[0] >> half
    ctr[0] &= mask
    ctr[2], ctr[3] = u(offset & 0xFFFFFFFF), u((offset >> 32) & 0xFFFFFFFF)
    for r in range(10):
        key = [u((seed + r * 0x9E3779B9) & 0xFFFFFFFF),
               u(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)]
        a, b = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = np.stack(((b >> half) ^ ctr[1] ^ key[0], b & mask,
                        (a >> half) ^ ctr[3] ^ key[1], a & mask))
    bits = ctr.T.astype(np.uint32).copy().view(np.uint16).reshape(-1)[:n]   # low half first
    return bits.astype(np.int64) >= int(math.floor(p * 65536 + 0.5))


def _exact_drop(s):
    keep = torch.from_numpy(_exact_keep(s["n"], s["p"], s["seed"], s["offset"])).cuda()
    T = int(math.floor(s["p"] * 65536 + 0.5))
    scale = 65536.0 / (65536 - T)
    y = s["res"].double() + s["x"].double() * keep * scale
    if s["kind"] == "drop":
        return y
    return y, s["dy"].double() * keep * scale


def _exact_attn(s):
    """One window and head at a time; the gradients by differentiation."""
    W, H, G, d = (s[k] for k in ("windows", "heads", "kv_heads", "d"))
    nq, nk, dv, grad = s["n_q"], s["n_k"], s["dv"], s["kind"] == "attn_grad"
    if W * H > 8192:
        return None                       # thousands of small products: too slow one by one
    q, k, v, lam = (s[n].double() for n in ("q", "k", "v", "lam"))
    lens = _lengths(s)
    o = torch.zeros(W, H, nq, dv, dtype=torch.float64, device=q.device)
    gq, gk, gv, gl = (torch.zeros_like(t) for t in (q, k, v, lam))
    rows, cols = torch.arange(nq, device=q.device)[:, None], torch.arange(nk, device=q.device)
    for w in range(W):
        for h in range(H):
            c = h // (H // G)
            ln = lens[w]
            last = {"none": rows * 0 + ln, "start": rows, "end": rows + ln - nq}[s["causal"]]
            see = (cols[:ln] <= last)
            leaf = [t.detach().clone().requires_grad_(grad) for t in
                    (q[w, 2 * h], q[w, 2 * h + 1], k[w, 2 * c, :ln], k[w, 2 * c + 1, :ln],
                     v[w, c, :ln], lam[h])]
            q1, q2, k1, k2, vv, l = leaf
            if ln == 0:
                continue
            bias = torch.zeros(nq, ln, dtype=torch.float64, device=q.device).masked_fill_(~see, -1e300)
            some = see.any(1, keepdim=True)
            maps = [torch.softmax(a @ b.t() / math.sqrt(d) + bias, -1) * some
                    for a, b in ((q1, k1), (q2, k2))]
            out = (maps[0] - l * maps[1]) @ vv
            o[w, h] = out.detach()
            if grad:
                a = torch.autograd.grad(out, leaf, s["do"][w, h].double())
                gq[w, 2 * h] += a[0]
                gq[w, 2 * h + 1] += a[1]
                gk[w, 2 * c, :ln] += a[2]
                gk[w, 2 * c + 1, :ln] += a[3]
                gv[w, c, :ln] += a[4]
                gl[h] += a[5]
    return (o, gq, gk, gv, gl) if grad else o


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"].split("_")[0]
    return {"norm": _exact_norm, "drop": _exact_drop, "attn": _exact_attn}[kind](s)
