"""Differential attention against its formulas in 64 bits: output and gradients at
the sizes, masks and layouts where a tile, a split or a store can go wrong."""
import pytest
import torch

from paper_2506_08520_amd import binding as B
import operators_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(W, H, G, nq, nk, d, dv, dtype, seed=0, tokens=False):
    g = torch.Generator().manual_seed(1000 * seed + 7 * nq + nk + d)

    def draw(*shape, mean=0.0):
        x = (torch.randn(*shape, generator=g) + mean).to(DT[dtype]).cuda()
        return x.transpose(1, 2).contiguous().transpose(1, 2) if tokens else x
    q, k, v = draw(W, 2 * H, nq, d), draw(W, 2 * G, nk, d), draw(W, G, nk, dv, mean=0.25)
    do = draw(W, H, nq, dv)
    lam = (0.1 + 0.8 * torch.rand(H, generator=g)).cuda()
    return q, k, v, lam, do


def lens(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def run(q, k, v, lam, do, causal=0, kv_len=None, scale=0.0, what=""):
    n = lens(kv_len)
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, scale=scale, causal=causal, kv_len=n,
                                          with_saved=True)
    only = B.nystra_diff_attn_forward(q, k, v, lam, scale=scale, causal=causal, kv_len=n)
    grads = B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved, scale=scale, causal=causal,
                                        kv_len=n)
    torch.cuda.synchronize()
    want = ref.diff_attention(*(t.cpu() for t in (q, k, v, lam)), causal=causal, kv_len=kv_len,
                              scale=scale or None, do=do.cpu())
    assert torch.equal(only, o)
    for got, pair, name in zip((o, *grads), want, ("O", "dQ", "dK", "dV", "dlam")):
        ref.check(got, pair, f"{what} {name}")
    return o, grads


# (W, H, G, nq, nk, d, dv, causal, kv_len, tokens)
SIZES = [
    (1, 1, 1, 1, 1, 1, 1, 0, None, False),
    (2, 1, 1, 1, 1, 30, 60, 0, None, False),
    (2, 2, 1, 2, 3, 5, 7, 0, None, True),
    (4, 6, 6, 64, 64, 30, 60, 0, None, True),        # a SwinIR window
    (3, 2, 2, 64, 64, 32, 64, 0, None, False),
    (2, 3, 3, 33, 47, 17, 37, 0, None, True),        # odd everything: element loads
    (1, 4, 2, 65, 95, 33, 65, 0, None, False),
    (1, 2, 2, 127, 256, 64, 128, 0, None, False),    # the longest with D from a first walk
    (1, 2, 2, 128, 257, 64, 128, 0, None, True),     # the shortest with stored outputs
    (2, 4, 2, 60, 256, 20, 61, 2, [256, 40], True),
    (2, 4, 2, 60, 258, 20, 61, 2, [258, 40], True),
    (2, 8, 2, 100, 100, 44, 88, 1, None, True),
    (1, 2, 1, 257, 257, 48, 96, 1, None, False),
    (2, 4, 2, 31, 200, 24, 128, 2, None, False),
    (4, 2, 2, 50, 50, 30, 60, 1, [50, 0, 1, 33], True),
    (5, 4, 2, 290, 290, 16, 32, 1, [290, 0, 1, 127, 1000], False),
    (5, 2, 1, 9, 150, 64, 100, 2, [150, 0, 4, 9, -3], False),   # rows that see no key
    (3, 3, 1, 70, 140, 8, 128, 0, [0, 140, 65], True),
    (2, 16, 4, 1, 300, 64, 128, 2, [300, 77], False),
    (1, 1, 1, 300, 2, 64, 3, 0, None, False),
    (1, 6, 6, 1, 197, 30, 60, 2, None, False),
    (1, 3, 3, 40, 33, 64, 4, 1, None, False),        # more queries than keys
    (4, 8, 2, 8, 1000, 64, 128, 2, [1000, 0, 1, 300], False),   # dQ by key ranges
    (3, 4, 2, 5, 777, 33, 61, 2, [3, 777, 500], True),
    (1, 2, 2, 300, 900, 21, 40, 1, None, False),
    (2, 8, 2, 1, 700, 46, 92, 2, [700, 33], False),      # rows of 4-byte groups, full width
    (1, 2, 2, 70, 300, 46, 90, 0, None, True),
    (2, 2, 1, 40, 50, 2, 2, 0, [50, 7], False),          # the narrowest of them
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(str(x) for x in s[:8]))
def test_output_and_gradients(size, dtype):
    W, H, G, nq, nk, d, dv, causal, kv_len, tokens = size
    run(*make(W, H, G, nq, nk, d, dv, dtype, tokens=tokens), causal=causal, kv_len=kv_len,
        what=f"{size} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 2, 1, 1, 4099, 64, 128), (2, 4, 2, 3, 2500, 30, 60),
                                  (1, 1, 1, 40, 1500, 16, 33)],
                         ids=lambda s: "x".join(map(str, s)))
def test_keys_split_over_workgroups(size, dtype):
    W, H, G, nq, nk, d, dv = size
    q, k, v, lam, do = make(*size, dtype)
    shape = B.DiffShape(W, H, G, nq, nk, d, dv, B.CAUSAL_END, 0.0)
    assert B.nystra_diff_attn_workspace_size(shape) > 0
    # One length ends inside a range, so that the last ranges hold nothing.
    run(q, k, v, lam, do, causal=B.CAUSAL_END, kv_len=[nk // 3 + 1] * W, what=f"split {size}")
    run(q, k, v, lam, do, causal=B.CAUSAL_END, what=f"split {size}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_keep_their_maximum(dtype):
    """Scores around +-1000: the exponent of each row is taken against its maximum."""
    q, k, v, lam, do = make(1, 2, 2, 70, 200, 16, 32, dtype)
    o = B.nystra_diff_attn_forward(q, k, v, lam, scale=100.0)
    want = ref.diff_attention(*(t.cpu() for t in (q, k, v, lam)), scale=100.0)
    ref.check(o, want[0], "large scores")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_maps_cancel(dtype):
    """With both maps equal and lam = 1 the output is exactly zero."""
    q, k, v, lam, _ = make(2, 2, 2, 64, 300, 32, 64, dtype)
    q[:, 1::2], k[:, 1::2] = q[:, ::2], k[:, ::2]
    o = B.nystra_diff_attn_forward(q, k, v, torch.ones_like(lam))
    assert (o == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nk", [40, 400])
def test_what_lies_behind_the_length_is_not_read(nk, dtype):
    """Infinities and NaN in keys and values behind the length change nothing, and
    their gradients are zero."""
    kv_len = [nk // 2 + 3, 0, 1]
    q, k, v, lam, do = make(3, 2, 1, 37, nk, 20, 40, dtype)
    o, grads = run(q, k, v, lam, do, kv_len=kv_len, what="clean")
    for w, n in enumerate(kv_len):
        k[w, :, n:], v[w, :, n:] = float("nan"), float("inf")
    o2, grads2 = run(q, k, v, lam, do, kv_len=kv_len, what="poisoned")
    assert torch.equal(o, o2)
    for a, b in zip(grads, grads2):
        assert torch.equal(a, b)
    for w, n in enumerate(kv_len):
        assert (grads2[1][w, :, n:] == 0).all() and (grads2[2][w, :, n:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_key_has_no_gradient_of_scores(dtype):
    """A softmax over one key is 1: dQ and dK vanish exactly."""
    q, k, v, lam, do = make(2, 2, 2, 5, 1, 30, 60, dtype)
    _, (dq, dk, _, _) = run(q, k, v, lam, do, what="one key")
    assert (dq == 0).all() and (dk == 0).all()


@pytest.mark.parametrize("nk", [150, 300])
def test_gradients_against_differences(nk):
    """Central differences of sum(O dO) along random directions, fp32 inputs: the
    slope of a 64-bit evaluation at points a step apart."""
    args = make(2, 4, 2, 12, nk, 10, 20, "f32")
    q, k, v, lam, do = args
    kv_len = [nk, nk - 19]
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, kv_len=lens(kv_len), causal=2,
                                          with_saved=True)
    grads = B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved, kv_len=lens(kv_len), causal=2)
    leaves = [t.cpu().double() for t in (q, k, v, lam)]
    g = torch.Generator().manual_seed(3)
    for i in range(4):
        u = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        f = []
        for sign in (1, -1):
            moved = [t + sign * h * u if j == i else t for j, t in enumerate(leaves)]
            f.append(float((value64(*moved, 2, kv_len) * do.cpu().double()).sum()))
        slope = (f[0] - f[1]) / (2 * h)
        got = float((grads[i].cpu().double() * u).sum())
        # fp32 gradients: rounding relative to the sum of magnitudes; the difference's own
        # error is of order h^2 and 1e-16 / h.
        tol = 2e-5 * float((grads[i].cpu().double() * u).abs().sum()) + 1e-7
        assert abs(slope - got) <= tol, (i, slope, got)


def value64(q, k, v, lam, causal, kv_len):
    W, H, R = q.shape[0], q.shape[1] // 2, q.shape[1] // 2 // v.shape[1]
    see = ref.visible(W, q.shape[2], v.shape[2], causal, kv_len)
    out = []
    for w in range(W):
        for h in range(H):
            c = h // R
            maps = [torch.softmax((q[w, 2 * h + a] @ k[w, 2 * c + a].t() / q.shape[3] ** 0.5)
                                  .masked_fill(~see[w], -1e300), -1) for a in range(2)]
            out.append((maps[0] - lam[h] * maps[1]) @ v[w, c])
    return torch.stack(out).reshape(W, H, *out[0].shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_of_fused_and_shared_buffers(dtype):
    """Q, K, V as column blocks of one projection, their gradients written into one
    buffer of the same layout; and values broadcast over the windows."""
    W, H, N, d, dv = 2, 3, 45, 10, 18
    width = 4 * H * d + H * dv
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(W, N, width, generator=g).to(DT[dtype]).cuda()
    gfused = torch.full_like(fused, float("nan"))

    def parts(t):
        a, b = 2 * H * d, 4 * H * d
        return (t[..., :a].unflatten(-1, (2 * H, d)).transpose(1, 2),
                t[..., a:b].unflatten(-1, (2 * H, d)).transpose(1, 2),
                t[..., b:].unflatten(-1, (H, dv)).transpose(1, 2))
    q, k, v = parts(fused)
    lam = torch.full((H,), 0.5, device="cuda")
    out = torch.empty(W, N, H, dv, dtype=DT[dtype], device="cuda").transpose(1, 2)
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, with_saved=True, out=out)
    do = torch.randn(o.shape, generator=g).to(DT[dtype]).cuda()
    B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved, grads=parts(gfused))
    want = ref.diff_attention(*(t.cpu() for t in (q, k, v, lam)), do=do.cpu())
    for got, pair, name in zip((out, *parts(gfused)), want, ("O", "dQ", "dK", "dV")):
        ref.check(got, pair, f"fused {name}")
    shared = v[:1].expand(W, H, N, dv)
    run(q, k, shared, lam, do, what="broadcast values")


def test_offsets_past_32_bits():
    """Keys and values of one long strided cache: tokens 2^22 elements apart."""
    nk, d, dv, step = 600, 16, 32, 1 << 22
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 6 GB of device memory")
    buf = torch.empty(nk * step, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(buf, (1, 2, nk, d), (0, 64, step, 1))
    v = torch.as_strided(buf, (1, 1, nk, dv), (0, 0, step, 1), 256)
    q, k0, v0, lam, do = make(1, 1, 1, 3, nk, d, dv, "bf16")
    k.copy_(k0)
    v.copy_(v0)
    o = B.nystra_diff_attn_forward(q, k, v, lam)
    o0, saved = B.nystra_diff_attn_forward(q, k0, v0, lam, with_saved=True)
    assert torch.equal(o, o0)
    near = B.nystra_diff_attn_backward(do, q, k0, v0, lam, o0, saved)
    far = B.nystra_diff_attn_backward(do, q, k, v, lam, o0, saved)
    for a, b in zip(near, far):
        assert torch.equal(a, b)


@pytest.mark.parametrize("nk", [64, 700])
def test_same_bits_every_time_and_on_any_stream(nk):
    q, k, v, lam, do = make(3, 4, 2, 64, nk, 30, 60, "bf16")
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, with_saved=True)
    grads = B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        o2, saved2 = B.nystra_diff_attn_forward(q, k, v, lam, with_saved=True, stream=side)
        grads2 = B.nystra_diff_attn_backward(do, q, k, v, lam, o2, saved2, stream=side)
        side.synchronize()
        assert torch.equal(o, o2)
        for a, b in zip(grads, grads2):
            assert torch.equal(a, b)


@pytest.mark.parametrize("size", [(8, 6, 6, 64, 64, 30, 60), (1, 4, 2, 2, 1500, 64, 128)],
                         ids=["window", "split"])
def test_graph_replays_equal_eager_calls(size):
    bufs = list(make(*size, "bf16"))
    n = torch.full((size[0],), size[4], dtype=torch.int32, device="cuda")

    def step(q, k, v, lam, do):
        o, saved = B.nystra_diff_attn_forward(q, k, v, lam, kv_len=n, causal=2, with_saved=True)
        return (o, *B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved, kv_len=n, causal=2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*bufs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*bufs)
    for rep in range(4):
        for b, x in zip(bufs, make(*size, "bf16", seed=10 + rep)):
            b.copy_(x)
        n.fill_(size[4] - 3 * rep)
        want = step(*bufs)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), rep


def test_no_windows():
    """The gradient of lambda over no windows is zero, everything else is empty."""
    q, k, v, lam, do = make(0, 4, 2, 8, 12, 16, 32, "f32")
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, with_saved=True)
    dq, dk, dv, dlam = B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved)
    assert o.shape == do.shape and dq.shape == q.shape and dk.shape == k.shape
    assert (dlam == 0).all()
