"""Group norm + activation over channels-last activations, element by element against the 64-bit reference.

Tolerances.  Sums run over chains of at most D = 256 additions (a thread's own, then trees), each off by 2^-24 of a partial sum:
a mean is off by at most D 2^-24 max|x|, a variance by 2 D 2^-24 of itself besides, so that before the activation
  |error| <= D 2^-24 (max|x - mean| + max|x|) rstd |gamma| + D 2^-24 |v - beta| + 8 * 2^-24 (|v| + |beta|).
The activations' slopes are at most 1.13, and their own evaluation is off by 2^-20 of the value.  bf16 results add 2^-8 of
themselves; the 8-bit ones 2^-4 of themselves, 2^-10 of the scale, and the scale's error once more.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import blocks as B
from paper_2201_05587_amd import api

F32, BF16 = api.TT_F32, api.TT_BF16
ACTS = (api.TT_ACT_NONE, api.TT_ACT_RELU, api.TT_ACT_RELU6, api.TT_ACT_GELU, api.TT_ACT_SILU)
D = 256


def make(seed, n, h, w, c, dtype, offset=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, h, w, c)) * np.exp(0.5 * rng.standard_normal(c)) + offset * rng.standard_normal(c)
    gamma, beta = 1 + 0.2 * rng.standard_normal(c), 0.2 * rng.standard_normal(c)
    return [torch.from_numpy(t.astype(np.float32)).to(api.torch_dtype(dtype)) for t in (x, gamma, beta)]


def reference(x, gamma, beta, groups, act, eps):
    """(y, tolerance) in 64 bits."""
    x, gamma, beta = (None if t is None else t.double().cpu().numpy() for t in (x, gamma, beta))
    y, v, rstd, mean = B.group_norm(x, gamma, beta, groups, act, eps)
    n, h, w, c = x.shape
    parts = lambda t: t.reshape(n, h * w, groups, c // groups)  # noqa: E731
    top = parts(np.abs(x - mean)).max(axis=(1, 3), keepdims=True) + parts(np.abs(x)).max(axis=(1, 3), keepdims=True)
    top = np.broadcast_to(top, parts(x).shape).reshape(x.shape)
    g, b = np.ones(c) if gamma is None else np.abs(gamma), np.zeros(c) if beta is None else beta
    tol = 2.0 ** -24 * (D * top * rstd * g + D * np.abs(v - b) + 8 * (np.abs(v) + np.abs(b)))
    return y, 1.13 * tol + 2.0 ** -20 * np.abs(y)


def check(n, h, w, c, groups, dtype, act, fp8=False, affine=True, eps=1e-5, offset=1.0, tensors=None):
    x, gamma, beta = tensors or make(n + h * 3 + w * 5 + c * 7, n, h, w, c, dtype, offset)
    if not affine:
        gamma = beta = None
    y, tol = reference(x, gamma, beta, groups, act, eps)
    shape = api.tt_norm_shape(n, h, w, c, groups, dtype)
    on = [None if t is None else t.cuda() for t in (x, gamma, beta)]
    rows, kb, guard = n * h * w, -(-c // 128), 128
    need = api.tt_norm_plan(shape, fp8).workspace_bytes
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    if not fp8:
        whole = torch.full((rows * c + 2 * guard,), float("nan"), dtype=api.torch_dtype(dtype), device="cuda")
        out = whole[guard:guard + rows * c].view(n, h, w, c)
        assert api.tt_group_norm_act(*on, shape, act, eps, ws=ws[:need], y=out) is out
        torch.cuda.synchronize()
        assert bool(torch.isnan(whole[:guard]).all()) and bool(torch.isnan(whole[guard + rows * c:]).all())
        got = out.double().cpu().numpy()
        if dtype == BF16:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(y)
    else:
        q = torch.full((rows * kb * 128 + 2 * guard,), 3.0, device="cuda").to(torch.float8_e4m3fn)
        s = torch.full((rows * kb + 2 * guard,), -7.0, device="cuda")
        nq, ns = rows * kb * 128, rows * kb
        api.tt_group_norm_act_fp8(*on, shape, act, eps, ws=ws[:need], q=q[guard:guard + nq], scale=s[guard:guard + ns])
        torch.cuda.synchronize()
        for t, v, size in ((q.float(), 3, nq), (s, -7, ns)):
            assert bool((t[:guard] == v).all()) and bool((t[guard + size:] == v).all())
        vals = q[guard:guard + nq].double().cpu().numpy().reshape(1, rows, kb * 128)
        scale = s[guard:guard + ns].double().cpu().numpy().reshape(1, kb, rows)
        assert not vals[:, :, c:].any()
        top = np.abs(np.pad(y.reshape(rows, c), ((0, 0), (0, kb * 128 - c)))).reshape(rows, kb, 128).max(axis=2)
        t2 = np.pad(tol.reshape(rows, c), ((0, 0), (0, kb * 128 - c))).reshape(rows, kb, 128).max(axis=2)
        assert (np.abs(scale[0].T - np.maximum(top, 2.0 ** -100) / 448) <= (t2 + 2.0 ** -22 * top) / 448 + 1e-40).all()
        got = B.dequantize(vals, scale, 1)[0][:, :c].reshape(n, h, w, c)
        wide = np.repeat(scale[0].T, 128, axis=1)[:, :c].reshape(n, h, w, c)
        tol = tol * (1 + 2.0 ** -4) + 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * wide + 2.0 ** -21 * np.abs(y)
    assert bool((ws[need:] == 255).all())
    err = np.abs(got - y)
    bad = ~(err <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float((err / tol).max()))


SIZES = [(1, 1, 1, 1, 1), (1, 1, 1, 32, 32), (3, 1, 1, 40, 8), (1, 9, 7, 90, 9), (2, 8, 8, 128, 32), (1, 5, 3, 130, 13), (2, 16, 16, 320, 32),
         (1, 33, 17, 96, 1), (4, 7, 7, 512, 32), (1, 1, 300, 72, 3), (2, 3, 3, 2048, 32), (1, 40, 40, 64, 64), (1, 31, 29, 1000, 8), (5, 64, 48, 24, 3),
         (1, 2, 2, 10240, 4), (1, 2, 5, 5001, 3), (1, 128, 130, 16, 2), (1, 2, 1, 2048, 2048),
         (1, 40, 30, 1000, 1000), (2, 28, 28, 128, 32), (1, 60, 60, 640, 32), (3, 50, 37, 2056, 8), (17, 28, 28, 128, 32), (40, 14, 13, 64, 16),
         (300, 3, 5, 40, 8), (70, 5, 5, 256, 2), (130, 20, 11, 24, 3), (33, 11, 40, 128, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,h,w,c,groups", SIZES)
def test_group_norm(n, h, w, c, groups, dtype, fp8):
    check(n, h, w, c, groups, dtype, ACTS[(n + h + w + c) % 5], fp8)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("affine", [True, False])
def test_activations_with_and_without_weights(act, affine, fp8):
    for dtype in (F32, BF16):
        check(2, 6, 5, 48, 6, dtype, act, fp8, affine)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_means_far_from_zero_and_groups_without_variance(dtype):
    check(1, 12, 12, 64, 8, dtype, api.TT_ACT_NONE, offset=300.0)
    check(1, 70, 70, 64, 8, dtype, api.TT_ACT_SILU, offset=300.0)
    x = torch.full((2, 10, 10, 32), 7.0).to(api.torch_dtype(dtype))
    ones, zeros = torch.ones(32).to(x.dtype), torch.zeros(32).to(x.dtype)
    y = api.tt_group_norm_act(x.cuda(), ones.cuda(), zeros.cuda(), api.tt_norm_shape(2, 10, 10, 32, 4, dtype), api.TT_ACT_NONE, 1e-5)
    assert not bool(y.any())  # exactly the mean


def around(offset, n, h, w, c, dtype):
    """Normal values about one mean, the same for every channel, so that a group's mean is `offset` of its deviations."""
    rng = np.random.default_rng(c + h)
    t = [offset + rng.standard_normal((n, h, w, c)), 1 + 0.2 * rng.standard_normal(c), 0.2 * rng.standard_normal(c)]
    return [torch.from_numpy(v.astype(np.float32)).to(api.torch_dtype(dtype)) for v in t]


# in one pass and in two, with groups of whole vectors and without, in several parts, and in column tiles that end inside a group
FAR = [(1, 12, 12, 64, 8), (1, 70, 70, 64, 8), (2, 5, 3, 90, 9), (1, 41, 37, 90, 9), (1, 200, 190, 24, 3), (1, 50, 37, 2056, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dtype,offset", [(F32, 30.0), (F32, -300.0), (BF16, 30.0)])
@pytest.mark.parametrize("n,h,w,c,groups", FAR)
def test_groups_whose_mean_is_many_deviations(n, h, w, c, groups, dtype, offset, fp8):
    check(n, h, w, c, groups, dtype, api.TT_ACT_NONE, fp8, tensors=around(offset, n, h, w, c, dtype))


@pytest.mark.parametrize("offset", [30.0, -300.0])
@pytest.mark.parametrize("n,h,w,c,groups", FAR[:2])
def test_means_of_squares_in_32_bits_would_not_do(n, h, w, c, groups, offset):
    """What the test above is there for: E[x^2] - E[x]^2 from float32 sums is outside its tolerance."""
    x, gamma, beta = around(offset, n, h, w, c, F32)
    y, tol = reference(x, gamma, beta, groups, api.TT_ACT_NONE, 1e-5)
    flat = x.numpy().reshape(n, h * w, groups, c // groups).transpose(0, 2, 1, 3).reshape(n, groups, -1)
    size = np.float32(flat.shape[2])
    mean = np.cumsum(flat, axis=2, dtype=np.float32)[..., -1] / size
    var = np.cumsum(flat * flat, axis=2, dtype=np.float32)[..., -1] / size - mean * mean
    spread = lambda t: np.repeat(t, c // groups, axis=1).reshape(n, 1, 1, c).astype(np.float64)  # noqa: E731
    with np.errstate(invalid="ignore"):
        naive = (x.double().numpy() - spread(mean)) / np.sqrt(spread(var) + 1e-5) * gamma.double().numpy() + beta.double().numpy()
    assert not (np.abs(naive - y) <= tol).all()


# An activation's own error.  GELU: test_fp8.py's bound.  SiLU, v / (1 + exp(-v)): a product, a sum, an exponential and a reciprocal of
# less than 2^-20 together, and the exponent, rounded with its constant, by 1.5 * 2^-24 of |v|; a reciprocal below 2^-126 is 0.
@pytest.mark.gpu
@pytest.mark.parametrize("h", [2, 8])  # in one pass, and in two
@pytest.mark.parametrize("act", [api.TT_ACT_GELU, api.TT_ACT_SILU])
def test_activations_over_their_range(act, h):
    """As the shift of values times zero."""
    v = np.concatenate([np.linspace(-20, 20, 2000), np.linspace(-150, 150, 993), [1e-30, -1e-30, 1e30, -1e30, 3e38, -3e38, -0.0]]).astype(np.float32)
    x, c = v.astype(np.float64), 1000
    if act == api.TT_ACT_GELU:
        tail = np.array([0.5 * abs(t) * math.erfc(abs(t) / math.sqrt(2.0)) for t in x])
        y = np.maximum(x, 0.0) - tail
        tol = 2.0 ** -20 * np.abs(y) + 1.3 * 2.0 ** -24 * np.minimum(x * x, 1e6) * tail + 2.0 ** -126
    else:
        with np.errstate(over="ignore"):
            y = x / (1.0 + np.exp(-x))
        tol = np.abs(y) * (2.0 ** -20 + 1.5 * 2.0 ** -24 * np.minimum(np.abs(x), 1e3)) + np.minimum(np.abs(x), 1e3) * 2.0 ** -126
    shape = api.tt_norm_shape(1, h, h, c, 1, F32)
    assert api.tt_norm_plan(shape).kernel == (api.TT_NORM_ONE_PASS if h == 2 else api.TT_NORM_TWO_PASS)
    some = make(1, 1, h, h, c, F32)[0].cuda()
    for i in range(0, len(v), c):
        got = api.tt_group_norm_act(some, torch.zeros(c, device="cuda"), torch.from_numpy(v[i:i + c]).cuda(), shape, act).view(h * h, c)
        assert bool((got == got[:1]).all())
        bad = ~(np.abs(got[0].double().cpu().numpy() - y[i:i + c]) <= tol[i:i + c])
        assert not bad.any(), (int(bad.sum()), v[i:i + c][bad][:8])


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("c,groups", [(1, 1), (2, 1), (3, 3), (5, 1), (6, 3), (7, 7), (9, 3), (11, 1), (12, 3), (13, 13), (14, 2), (15, 5), (17, 1), (23, 1),
                                      (129, 3), (131, 1), (258, 6), (1003, 17)])
def test_rows_that_end_inside_an_item(c, groups, fp8):
    """In one pass and in two; rows shorter than an item of 16 bytes, and every length behind one."""
    for dtype in (F32, BF16):
        for n, h, w in ((1, 1, 1), (2, 5, 4), (2, 41, 37), (300, 3, 3)):
            check(n, h, w, c, groups, dtype, ACTS[(h + c) % 5], fp8, affine=h != 5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("h", [3, 64])
@pytest.mark.parametrize("c,groups", [(15, 3), (6, 2), (90, 9)])
def test_what_is_not_finite_stays_in_its_group_where_rows_end_inside_an_item(c, groups, h, dtype):
    x, gamma, beta = make(1, 3, h, h, c, dtype)
    wide = c // groups
    x[0, 0, 0, wide - 1], x[1, 1, 2, c - 1], x[2, 0, 1, wide] = float("nan"), float("nan"), float("inf")
    y = api.tt_group_norm_act(x.cuda(), gamma.cuda(), beta.cuda(), api.tt_norm_shape(3, h, h, c, groups, dtype), api.TT_ACT_NONE, 1e-5).cpu()
    lost = torch.isnan(y).view(3, h * h, groups, wide)
    want = torch.zeros(3, groups, dtype=torch.bool)
    want[0, 0] = want[1, groups - 1] = want[2, 1] = True
    assert torch.equal(lost.any(dim=3).any(dim=1), want)
    assert bool(lost[1, :, groups - 1].all())


@pytest.mark.gpu
@pytest.mark.parametrize("h", [3, 64])
def test_what_is_not_finite_stays_in_its_image_and_group(h):
    x, gamma, beta = make(1, 3, h, h, 64, F32)
    x[1, 1, 2, 20], x[2, 0, 1, 40] = float("nan"), float("inf")
    y = api.tt_group_norm_act(x.cuda(), gamma.cuda(), beta.cuda(), api.tt_norm_shape(3, h, h, 64, 4, F32), api.TT_ACT_SILU, 1e-5).cpu()
    lost = torch.isnan(y).view(3, h * h, 4, 16)
    want = torch.zeros(3, 4, dtype=torch.bool)
    want[1, 1] = want[2, 2] = True
    assert torch.equal(lost.any(dim=3).any(dim=1), want)
    assert bool(lost[1, :, 1].all())


@pytest.mark.gpu
def test_group_norm_is_the_same_every_time_on_every_stream_and_in_a_graph():
    for n, h, c, groups, dtype in ((1, 8, 96, 8, F32), (2, 64, 320, 32, BF16), (8, 32, 256, 32, BF16)):
        x, gamma, beta = (t.cuda() for t in make(n, n, h, h, c, dtype))
        shape = api.tt_norm_shape(n, h, h, c, groups, dtype)
        need = max(16, api.tt_norm_plan(shape).workspace_bytes, api.tt_norm_plan(shape, True).workspace_bytes)
        want = api.tt_group_norm_act(x, gamma, beta, shape, api.TT_ACT_SILU)
        want_q, want_s = api.tt_group_norm_act_fp8(x, gamma, beta, shape, api.TT_ACT_SILU)
        torch.cuda.synchronize()
        outs = []
        for s in [torch.cuda.Stream() for _ in range(2)]:
            with torch.cuda.stream(s):
                ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
                outs.append((api.tt_group_norm_act(x, gamma, beta, shape, api.TT_ACT_SILU, ws=ws), ws))
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o, _ in outs)
        y, q, s, ws = torch.empty_like(want), torch.empty_like(want_q), torch.empty_like(want_s), torch.empty(need, dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            api.tt_group_norm_act(x, gamma, beta, shape, api.TT_ACT_SILU, ws=ws, y=y)
            api.tt_group_norm_act_fp8(x, gamma, beta, shape, api.TT_ACT_SILU, ws=ws, q=q, scale=s)
        for _ in range(3):
            y.fill_(float("nan")), s.fill_(float("nan")), ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(s, want_s) and torch.equal(q.view(torch.uint8), want_q.view(torch.uint8))


@pytest.mark.gpu
def test_maps_beyond_32_bit_offsets():
    n, h, w, c, groups = 3, 1300, 1300, 512, 32  # 2.6e9 elements, in more parts than a small map's
    x = torch.empty(n, h, w, c, dtype=torch.bfloat16, device="cuda")
    for i in range(n):
        x[i].normal_()
    shape = api.tt_norm_shape(n, h, w, c, groups, BF16)
    y = api.tt_group_norm_act(x, None, None, shape, api.TT_ACT_NONE, 0.0)
    part = x[2, :, :, 480:].double()
    want = (part - part[..., 16:].mean()) / part[..., 16:].var(correction=0).sqrt()
    err = (y[2, :, :, 496:].double() - want[..., 16:]).abs()
    assert bool((err <= 2.0 ** -8 * want[..., 16:].abs() + D * 2.0 ** -23 * 12).all())


# ---- the operators one after the other ----------------------------------------------------------------------------------
@pytest.mark.gpu
def test_convolution_norm_and_8_bit_product_one_after_the_other():
    """A convolution of the library, group norm + SiLU written as 8-bit blocks, and the 8-bit pointwise product with bias and
    ReLU, as a network runs them: every step against the reference on that step's own input."""
    from oracle import ops as O
    from paper_2201_05587_amd import workloads as wl
    rng = np.random.default_rng(11)
    n, h, w, c, k, groups = 2, 12, 10, 48, 200, 8
    conv = wl.ConvShape(n, 16, h, w, c, 3, 3, 1, 1, 1, 1, wl.BF16)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16()  # noqa: E731
    x, f, bias = bf(rng.standard_normal((n, h, w, 16))), bf(rng.standard_normal((c, 3, 3, 16)) / 12), bf(rng.standard_normal(c))
    gamma, beta, wide, b2 = bf(1 + 0.2 * rng.standard_normal(c)), bf(0.2 * rng.standard_normal(c)), bf(rng.standard_normal((k, c)) / 7), bf(rng.standard_normal(k))
    t1 = api.tt_conv2d_bias_relu(x.cuda(), f.cuda(), bias.cuda(), None, conv, wl.CLS_CONV2D_ADD)  # (made as [n, k, Ho, Wo], stored channels-last)
    t1 = t1.reshape(n, h, w, c)
    q, s = api.tt_group_norm_act_fp8(t1, gamma.cuda(), beta.cuda(), api.tt_norm_shape(n, h, w, c, groups, BF16), api.TT_ACT_SILU, 1e-5)
    qw, sw = api.tt_quantize_fp8(wide.cuda(), api.tt_quant_shape(1, k, c, 128, BF16))
    y = api.tt_dense_fp8(q, s, qw, sw, b2.cuda(), api.tt_fp8_shape(1, n * h * w, k, c, 128, BF16), api.TT_DENSE_BIAS_RELU)
    ref = O.conv2d(*(t.float().numpy().transpose(0, 3, 1, 2).copy() for t in (x, f)), bias.float().numpy(), None, (1, 1), (1, 1), O.ACT_NONE)
    assert np.abs(t1.float().cpu().numpy().transpose(0, 3, 1, 2) - ref).max() <= 2e-2 * np.abs(ref).max()
    v, tol = reference(t1, gamma, beta, groups, api.TT_ACT_SILU, 1e-5)
    got = B.dequantize(q.double().cpu().numpy()[None], s.double().cpu().numpy()[None], 1)[0][:, :c].reshape(v.shape)
    unit = np.repeat(s.double().cpu().numpy().T, 128, axis=1)[:, :c].reshape(v.shape)
    assert (np.abs(got - v) <= tol * (1 + 2.0 ** -4) + (2.0 ** -4 + 2.0 ** -21) * np.abs(v) + 2.0 ** -10 * unit).all()
    want_q, want_s = B.quantize(wide.float().numpy()[None], 128)
    assert np.array_equal(qw.float().cpu().numpy(), want_q) and np.array_equal(sw.cpu().numpy(), want_s)
    p, size = B.product(q.double().cpu().numpy()[None], s.cpu().numpy()[None], want_q, want_s, 128)
    b2 = b2.double().numpy()
    want = np.maximum(p[0] + b2, 0)
    assert (np.abs(y.double().cpu().numpy() - want) <= 8 * 2.0 ** -13 * (size[0] + np.abs(b2)) * (1 + 2.0 ** -4) + 2.0 ** -8 * want).all()


def test_the_plan_of_a_group_norm():
    plan = lambda *a, fp8=False: api.tt_norm_plan(api.tt_norm_shape(*a), fp8)  # noqa: E731
    for fp8 in (False, True):
        assert plan(1, 3, 3, 64, 8, F32, fp8=fp8).kernel == api.TT_NORM_ONE_PASS and plan(1, 3, 3, 64, 8, F32, fp8=fp8).workspace_bytes == 0
        p = plan(2, 64, 64, 320, 32, BF16, fp8=fp8)
        assert p.kernel == api.TT_NORM_TWO_PASS and 1 <= p.chunks <= 64 and p.workspace_bytes == 2 * 32 * p.chunks * 8
    # a part is never longer than float32 sums over 128 batches of four pixels a thread allow
    p = plan(1, 1 << 15, 1 << 15, 1, 1, BF16)
    assert p.kernel == api.TT_NORM_TWO_PASS and p.chunks * 512 * 4 * 128 >= 1 << 30 and p.workspace_bytes == p.chunks * 8


# ---- refusals (no GPU is reached) ------------------------------------------------------------------------------------
def at(k=1):
    return ctypes.c_void_p(4096 * k)


def test_group_norm_refuses_what_is_ill_formed():
    bad = api.TT_ERR_BAD_ARG
    good = dict(n=2, h=3, w=3, c=12, groups=4, dtype=F32)

    def call(s, fp8=False, x=at(1), gamma=at(2), beta=at(3), y=at(4), scale=at(5), act=0, eps=1e-5, ws=at(6), ws_bytes=1 << 20):
        s = None if s is None else ctypes.byref(s)
        if fp8:
            return api.lib.tt_group_norm_act_fp8(x, gamma, beta, y, scale, s, act, eps, ws, ws_bytes, None)
        return api.lib.tt_group_norm_act(x, gamma, beta, y, s, act, eps, ws, ws_bytes, None)

    for fp8 in (False, True):
        for change in (dict(n=0), dict(h=0), dict(w=-1), dict(c=0), dict(groups=0), dict(groups=5), dict(groups=24), dict(dtype=3)):
            assert call(api.tt_norm_shape(**{**good, **change}), fp8) == bad, change
        s = api.tt_norm_shape(**good)
        for change in (dict(x=None), dict(y=None), dict(x=ctypes.c_void_p(4)), dict(gamma=ctypes.c_void_p(4100)), dict(act=5), dict(act=-1),
                       dict(eps=-1.0), dict(eps=float("nan"))):
            assert call(s, fp8, **change) == bad, change
        assert call(None, fp8) == bad
        big = api.tt_norm_shape(2, 64, 64, 320, 32, BF16)
        need = api.tt_norm_plan(big, fp8).workspace_bytes
        assert need > 0
        assert call(big, fp8, ws=None) == api.TT_ERR_WORKSPACE
        assert call(big, fp8, ws_bytes=need - 1) == api.TT_ERR_WORKSPACE
        assert call(big, fp8, ws=ctypes.c_void_p(4104)) == api.TT_ERR_WORKSPACE
        assert call(api.tt_norm_shape(1 << 10, 1 << 10, 1 << 12, 128, 1, BF16), fp8) == api.TT_ERR_UNSUPPORTED
    assert call(api.tt_norm_shape(**good), True, scale=None) == bad
    assert api.lib.tt_norm_plan(None, 0, None) == bad


@pytest.mark.gpu
def test_the_binding_refuses_other_types_sizes_and_strides():
    x, gamma, beta = (t.cuda() for t in make(1, 2, 4, 4, 32, BF16))
    shape = api.tt_norm_shape(2, 4, 4, 32, 4, BF16)
    assert api.tt_group_norm_act(x, gamma, beta, shape).shape == x.shape
    for wrong in ((x.float(), gamma, beta), (x.permute(0, 3, 1, 2), gamma, beta), (x[:1], gamma, beta), (x, gamma.float(), beta), (x, gamma, beta[:16]),
                  (x.cpu(), gamma, beta)):
        with pytest.raises(api.TTError) as e:
            api.tt_group_norm_act(*wrong, shape)
        assert e.value.status == api.TT_ERR_BAD_ARG
    with pytest.raises(api.TTError):
        api.tt_group_norm_act(x, gamma, beta, shape, y=torch.empty_like(x).float())
