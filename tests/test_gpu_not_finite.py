"""Differential attention with values that are not finite: NaN where the formulas have it
and nowhere else, however the keys are divided over workgroups."""
import pytest
import torch

from paper_2506_08520_amd import binding as B
import operators_oracle as ref
from test_gpu_diff_attn import lens, make

pytestmark = pytest.mark.gpu

NAN = float("nan")


def call(q, k, v, lam, do, **kw):
    o, saved = B.nystra_diff_attn_forward(q, k, v, lam, with_saved=True, **kw)
    grads = B.nystra_diff_attn_backward(do, q, k, v, lam, o, saved, **kw)
    only = B.nystra_diff_attn_forward(q, k, v, lam, **kw)
    torch.cuda.synchronize()
    assert torch.equal(only.isnan(), o.isnan())
    return [t.cpu() for t in (o, *grads)]


def same_nan(got, want, name, more=False):
    bad = want.isnan() & ~got.isnan() if more else got.isnan() != want.isnan()
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0]}"


def compare(ts, clean, got, what, more=()):
    """NaN in the elements where the formulas in 64 bits have it (of the results in `more`
    also in others); what is finite is that of the same inputs without NaN, within the bounds
    of that call."""
    q, k, v, lam, do = (t.cpu() for t in ts)
    want = ref.diff_attention(q, k, v, lam, do=do)
    bounds = ref.diff_attention(*(t.cpu() for t in clean[:4]), do=clean[4].cpu())
    for x, (y, _), (z, e), name in zip(got, want, bounds, ("O", "dQ", "dK", "dV", "dlam")):
        same_nan(x, y, f"{what} {name}", name in more)
        ok = ~y.isnan() & ~x.isnan()
        assert ((x.double() - z).abs() <= e)[ok].all(), f"{what} {name}"


# One workgroup to a row's keys; up to eight key ranges; more than eight.
SPLITS = [(3, 4, 2, 70, 90), (2, 4, 2, 3, 200), (2, 4, 2, 1, 1000)]


@pytest.mark.parametrize("dtype,d,dv", [("f32", 30, 60), ("bf16", 30, 60), ("bf16", 32, 64),
                                        ("bf16", 31, 61), ("bf16", 64, 128), ("f32", 44, 88)])
@pytest.mark.parametrize("W,H,G,nq,nk", SPLITS)
@pytest.mark.parametrize("where", ["query", "query2", "key", "keys", "value"])
def test_nan(W, H, G, nq, nk, dtype, d, dv, where):
    clean = make(W, H, G, nq, nk, d, dv, dtype)
    q, k, v, lam, do = (t.clone() for t in clean)
    if where == "query":       # first map of head 1
        q[1, 2, nq // 2, d - 1] = NAN
    elif where == "query2":    # second map of head 2
        q[0, 5, nq - 1, 0] = NAN
    elif where == "key":
        k[1, 0, nk // 2, 3] = NAN
    elif where == "keys":      # one key range and more of them
        k[0, 3, 32:64] = NAN
    else:
        v[1, 1, nk - 1, dv - 1] = NAN
    ts = (q, k, v, lam, do)
    # fp32 forms D_1 from O, into which the second map's NaN went
    more = ("dQ", "dK") if dtype == "f32" and where in ("query2", "keys") else ()
    compare(ts, clean, call(*ts), f"{where} {dtype} {nq}x{nk}", more)


@pytest.mark.parametrize("dtype,d,dv", [("f32", 30, 60), ("bf16", 30, 60), ("bf16", 31, 61)])
@pytest.mark.parametrize("nq", [70, 300])
def test_nan_of_a_row_with_one_key(nq, dtype, d, dv):
    """A softmax over one NaN score is NaN, and so is the gradient of its key."""
    q, k, v, lam, do = make(2, 1, 1, nq, nq, d, dv, dtype)
    q[1, 0, 0, 5] = NAN
    o, dq, dk, dv_, dlam = call(q, k, v, lam, do, causal=B.CAUSAL_START)
    assert o[1, 0, 0].isnan().all() and not o[1, 0, 1:].isnan().any()
    assert dq[1, 0, 0].isnan().all() and not dq[1, 0, 1:].isnan().any()
    assert dk[1, 0, 0].isnan().all() and dv_[1, 0, 0].isnan().all()
    assert not any(t[0].isnan().any() for t in (o, dq, dk, dv_))


@pytest.mark.parametrize("dtype,d,dv", [("f32", 30, 60), ("bf16", 30, 60), ("bf16", 32, 64),
                                        ("bf16", 31, 61), ("bf16", 64, 128)])
@pytest.mark.parametrize("nq,nk,kv_len", [(40, 40, [25, 40, 0]), (70, 300, [1, 300, 69]),
                                          (9, 600, [8, 0, 3])])
def test_queries_without_keys_pass_no_gradient(nq, nk, kv_len, dtype, d, dv):
    """Rows in front of a sequence that is shorter than the queries: whatever they and their
    gradients hold, the results are those of zeros there."""
    kw = dict(causal=B.CAUSAL_END, kv_len=lens(kv_len))
    q, k, v, lam, do = make(3, 4, 2, nq, nk, d, dv, dtype)
    q2, do2 = q.clone(), do.clone()
    for w, n in enumerate(kv_len):
        unseen = max(0, nq - n)
        q[w, :, :unseen], do[w, :, :unseen] = 0, 0
        q2[w, :, :unseen:2], q2[w, :, 1:unseen:2] = NAN, float("inf")
        do2[w, :, :unseen] = NAN
    want, got = call(q, k, v, lam, do, **kw), call(q2, k, v, lam, do2, **kw)
    for x, y, name in zip(got, want, ("O", "dQ", "dK", "dV", "dlam")):
        assert torch.equal(x, y), name
        assert torch.isfinite(y).all(), name


@pytest.mark.parametrize("d,dv", [(31, 61), (64, 128)])
@pytest.mark.parametrize("nq,nk", [(70, 90), (3, 200), (40, 300)])
def test_minus_infinity_scores_in_bf16(nq, nk, d, dv):
    """A key of -inf against positive queries has the probability zero at any width; only the
    gradient of the queries meets it again, as 0 x inf in its column."""
    q, k, v, lam, do = make(2, 2, 1, nq, nk, d, dv, "bf16")
    q[..., d - 1] = q[..., d - 1].abs() + 0.5
    k[1, 0, nk // 3, d - 1] = -float("inf")
    k[1, 1, nk // 3, d - 1] = -float("inf")
    k[1, 1, nk - 1, d - 1] = -float("inf")
    o, dq, dk, dv_, dlam = call(q, k, v, lam, do)
    cpu = [t.cpu() for t in (q, k, v, lam, do)]
    want = ref.diff_attention(*cpu[:4], do=cpu[4])
    same_nan(dq, want[1][0], "dQ")
    finite = dq[..., :d - 1]
    assert torch.isfinite(finite).all()
    # The bounds are those of the call with zeros for the infinities.  A probability of zero
    # has no error; the others grow by 1 / (1 - P) of at most two keys' shares, below 2 where
    # P < 1/2: the scores are within a few units and the keys 90 at least.
    cpu[1] = torch.where(cpu[1].isinf(), 0, cpu[1])
    bound = ref.diff_attention(*cpu[:4], do=cpu[4])
    assert ((o.double() - want[0][0]).abs() <= 2 * bound[0][1]).all()
    assert torch.isfinite(dk).all() and torch.isfinite(dv_).all() and torch.isfinite(dlam).all()
