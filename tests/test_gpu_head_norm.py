"""Norm of heads with rotation and its gradient against 64 bits, and the gradient against differences."""
import numpy as np
import pytest
import torch

from oracle import kv_ref as K
from paper_2302_12510_amd import binding as B
from kv_util import DTYPES, inside_larger, typed, within

pytestmark = pytest.mark.gpu


def rotation(rng, rows, pairs):
    angle = rng.uniform(-7, 7, (rows, pairs))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def case(rng, T, Hq, Hkv, D, rot, dtype, rows=50):
    q, q64 = typed(rng.standard_normal((T, Hq, D)) * 2.0 ** rng.integers(-4, 5, (T, Hq, 1)), dtype)
    k, k64 = typed(rng.standard_normal((T, Hkv, D)), dtype)
    w = [rng.uniform(0.2, 2, D).astype(np.float32) for _ in range(2)]
    cos, sin = rotation(rng, rows, rot // 2)
    positions = rng.integers(0, rows, T)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return (q, k, dev(w[0]), dev(w[1]), dev(positions), dev(cos), dev(sin)), (q64, k64, w, cos.astype(np.float64)[positions], sin.astype(np.float64)[positions])


def check(args, ref, dtype, neighbours, eps=1e-6, back=True, rng=None, wrap=lambda t: t):
    q, k, wq, wk, positions, cos, sin = args
    q64, k64, w, c, s = ref
    q, k = wrap(q), wrap(k)
    got = B.dybit_head_norm_rope(q, k, wq, wk, positions, cos, sin, eps, neighbours)
    for g, x, wt in zip(got, (q64, k64), w):
        within(g, *K.head_norm_rope(x, wt.astype(np.float64), c, s, eps, neighbours, dtype))
    if not back:
        return
    (gq, gq64), (gk, gk64) = (typed(rng.standard_normal(x.shape), dtype) for x in (q64, k64))
    dq, dk, dwq, dwk = B.dybit_head_norm_rope_bwd(wrap(gq), wrap(gk), q, k, wq, wk, positions, cos, sin, eps, neighbours)
    for g, x, wt, dx, dw in ((gq64, q64, w[0], dq, dwq), (gk64, k64, w[1], dk, dwk)):
        wx, bx, ww, bw = K.head_norm_rope_bwd(g, x, wt.astype(np.float64), c, s, eps, neighbours, dtype)
        within(dx, wx, bx, "dx")
        within(dw, ww, bw, "dw")
    assert B.dybit_get_last_async_error() == B.OK


@pytest.mark.parametrize("D,rot", [(64, 64), (128, 128), (128, 96), (256, 256), (80, 80), (96, 96), (128, 74), (128, 2), (512, 512), (2, 2), (6, 4), (130, 18), (512, 100)])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_sizes(D, rot, dtype, neighbours):
    rng = np.random.default_rng(D + rot)
    check(*case(rng, 5, 6, 2, D, rot, dtype), dtype, neighbours, rng=rng)


@pytest.mark.parametrize("T", [1, 2, 3, 17, 1000, 2100, 4100])
@pytest.mark.parametrize("heads", [(1, 1), (7, 3), (32, 8)])
def test_tokens_and_heads(T, heads):
    rng = np.random.default_rng(T)
    check(*case(rng, T, *heads, 64, 64, "fp32"), "fp32", False, rng=rng)


@pytest.mark.parametrize("pad", [0, 1, 2, 4, 8])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strides(pad, dtype):
    rng = np.random.default_rng(pad)
    check(*case(rng, 9, 5, 2, 64, 32, dtype), dtype, False, rng=rng, wrap=lambda t: inside_larger(t, pad=pad))


def test_queries_alone_in_place_and_another_stream():
    rng = np.random.default_rng(1)
    args, _ = case(rng, 33, 4, 2, 128, 128, "bf16")
    q, k, wq, wk, positions, cos, sin = args
    want = B.dybit_head_norm_rope(*args)
    alone, none = B.dybit_head_norm_rope(q, None, wq, None, positions, cos, sin)
    assert none is None and torch.equal(alone, want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    qkv = torch.cat((q, k, k), 1)
    views = (qkv[:, :4], qkv[:, 4:6])
    side.wait_stream(torch.cuda.current_stream())
    got = B.dybit_head_norm_rope(*views, wq, wk, positions, cos, sin, out=views, stream=side)
    side.synchronize()
    assert got[0] is views[0] and torch.equal(qkv[:, :4], want[0]) and torch.equal(qkv[:, 4:6], want[1]) and torch.equal(qkv[:, 6:], k)
    g = [torch.randn_like(t) for t in (q, k)]
    want = B.dybit_head_norm_rope_bwd(*g, *args)
    again = B.dybit_head_norm_rope_bwd(*g, *args, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))                       # the sums have one order
    got = B.dybit_head_norm_rope_bwd(*g, *args, out=tuple(g))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    dq, dk, dwq, dwk = B.dybit_head_norm_rope_bwd(want[0], None, q, None, wq, None, positions, cos, sin)
    assert dk is None and dwk is None and torch.equal(dq, B.dybit_head_norm_rope_bwd(want[0], want[1], *args)[0])


def test_gradient_against_differences():
    """d(sum g y) along random directions, from the forward in 64 bits."""
    rng = np.random.default_rng(2)
    args, (q64, k64, w, c, s) = case(rng, 6, 3, 2, 64, 48, "fp32")
    (gq, gq64), (gk, gk64) = (typed(rng.standard_normal(x.shape), "fp32") for x in (q64, k64))
    dq, dk, dwq, dwk = B.dybit_head_norm_rope_bwd(gq, gk, *args, 1e-5, True)
    for x, wt, g, dx, dw in ((q64, w[0], gq64, dq, dwq), (k64, w[1], gk64, dk, dwk)):
        f = lambda x, wt: (g * K.head_norm_rope(x, wt, c, s, 1e-5, True, "fp32")[0]).sum()  # noqa: E731
        wt = wt.astype(np.float64)
        for _ in range(3):
            u, v = rng.standard_normal(x.shape), rng.standard_normal(wt.shape)
            h = 1e-5
            slope = (f(x + h * u, wt + h * v) - f(x - h * u, wt - h * v)) / (2 * h)
            got = (dx.double().cpu().numpy() * u).sum() + (dw.double().cpu().numpy() * v).sum()
            # second derivatives of the norm are of the order of the terms over the square of the row: h^2 of them is far below this
            assert abs(got - slope) <= 1e-5 * (np.abs(dx.double().cpu().numpy() * u).sum() + np.abs(dw.double().cpu().numpy() * v).sum())


def test_rows_of_zeros_and_extreme_size():
    rng = np.random.default_rng(3)
    args, (q64, k64, w, c, s) = case(rng, 4, 2, 2, 64, 64, "fp32")
    q = args[0]
    q[0] = 0
    q[1] *= 1e15
    q[2] *= 1e-15
    check(args, (q.double().cpu().numpy(), k64, w, c, s), "fp32", False, rng=rng, back=False)
    out = B.dybit_head_norm_rope(*args, 1e-6)[0]
    assert (out[0] == 0).all()


def test_positions_outside_the_table():
    rng = np.random.default_rng(4)
    args, _ = case(rng, 5, 2, 1, 64, 64, "bf16")
    want = B.dybit_head_norm_rope(*args)
    g = [torch.randn_like(t) for t in args[:2]]
    keep = torch.tensor([0, 2, 4], device="cuda")
    dwant = B.dybit_head_norm_rope_bwd(*(t[keep] for t in g), *(t[keep] for t in args[:2]), *args[2:4], args[4][keep], *args[5:])
    args[4][1], args[4][3] = -1, 50
    got = B.dybit_head_norm_rope(*args)
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    for a, b in zip(got, want):
        assert a[[1, 3]].isnan().all() and torch.equal(a[keep], b[keep])
    dgot = B.dybit_head_norm_rope_bwd(*g, *args)
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    for a, b in zip(dgot[:2], dwant[:2]):
        assert a[[1, 3]].isnan().all() and torch.equal(a[keep], b)
    for a, b in zip(dgot[2:], dwant[2:]):
        torch.testing.assert_close(a, b, rtol=1e-5, atol=1e-4)


def test_no_tokens():
    rng = np.random.default_rng(5)
    args, _ = case(rng, 0, 2, 1, 64, 64, "fp32")
    assert B.dybit_head_norm_rope(*args)[0].shape == (0, 2, 64)
    out = B.dybit_head_norm_rope_bwd(*(torch.randn_like(t) for t in args[:2]), *args)
    assert (out[2] == 0).all() and (out[3] == 0).all()


def test_refusals():
    rng = np.random.default_rng(6)
    q, k, wq, wk, positions, cos, sin = case(rng, 4, 2, 1, 64, 64, "fp32")[0]

    def refused(status, *args, **kw):
        with pytest.raises(B.DybitError) as e:
            B.dybit_head_norm_rope(*args, **kw)
        assert e.value.status == status

    refused(B.ERR_INVALID_ARG, q, k.half(), wq, wk, positions, cos, sin)
    refused(B.ERR_INVALID_ARG, q, k[:3], wq, wk, positions, cos, sin)
    refused(B.ERR_INVALID_ARG, q, k, wq, wk, positions, cos, sin, -1.0)
    refused(B.ERR_INVALID_ARG, q, k, wq, wk, positions, cos, sin, float("nan"))
    refused(B.ERR_INVALID_ARG, q[..., :32].contiguous(), None, wq[:32], None, positions, cos, sin)          # more pairs than a head has
    refused(B.ERR_INVALID_ARG, q, None, wq, None, positions, cos[:, :0].contiguous(), sin[:, :0].contiguous())
    with pytest.raises(TypeError):
        B.dybit_head_norm_rope(q, k, wq, wk, positions.int(), cos, sin)
    with pytest.raises(ValueError):
        B.dybit_head_norm_rope(q, k, wq, wk, positions[:3], cos, sin)
    with pytest.raises(ValueError):
        B.dybit_head_norm_rope(q.cpu(), k, wq, wk, positions, cos, sin)
    with pytest.raises(ValueError):
        B.dybit_head_norm_rope(q, k, wq[:5], wk, positions, cos, sin)
    with pytest.raises(ValueError):
        B.dybit_head_norm_rope(q.transpose(1, 2), k, wq, wk, positions, cos, sin)


@pytest.mark.parametrize("D,rot", [(64, 46), (80, 26), (96, 54), (128, 70), (256, 178), (512, 290), (64, 18), (96, 78), (34, 34), (50, 18)])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotations_of_odd_widths(D, rot, dtype, neighbours):
    """Pairs whose number the vector accesses do not divide, in heads that start anywhere, and in place."""
    rng = np.random.default_rng(D * 1000 + rot)
    args, ref = case(rng, 37, 7, 3, D, rot, dtype)
    check(args, ref, dtype, neighbours, rng=rng, wrap=lambda t: inside_larger(t, pad=D % 3 + 1))
    q, k, wq, wk, positions, cos, sin = args
    gq, gk = (torch.randn(x.shape, generator=torch.Generator().manual_seed(rot)).to(x.dtype).cuda() for x in (q, k))
    want = B.dybit_head_norm_rope(*args, 1e-6, neighbours), B.dybit_head_norm_rope_bwd(gq, gk, *args, 1e-6, neighbours)
    mine = q.clone(), k.clone()
    B.dybit_head_norm_rope(*mine, wq, wk, positions, cos, sin, 1e-6, neighbours, out=mine)
    assert all(torch.equal(a, b) for a, b in zip(mine, want[0]))


def test_an_infinite_element_of_overlapping_accesses():
    """An infinite element makes its own head's elements zero or NaN as the formula does, whichever access reads it, and no other head's."""
    rng = np.random.default_rng(11)
    for at in range(64):
        (q, k, wq, wk, positions, cos, sin), _ = case(rng, 2, 2, 1, 64, 46, "fp32")
        q[0, 1, at] = float("inf")
        got = B.dybit_head_norm_rope(q, k, wq, wk, positions, cos, sin)[0]
        clean = torch.isfinite(got[0, 1])
        touched = {at, at + 23 if at < 23 else at - 23 if at < 46 else at}
        assert {int(i) for i in torch.nonzero(~clean)} == touched and bool((got[0, 1][clean] == 0).all())
        assert bool(torch.isfinite(got[0, 0]).all() and torch.isfinite(got[1]).all())
