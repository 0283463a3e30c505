"""The 64-bit reference of the 8-bit block operators and of group norm, against torch on the CPU and against itself."""
import numpy as np
import pytest
import torch

from oracle import blocks as B


def test_e4m3_is_torchs_rounding():
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 6, 20000),
                        np.arange(-896, 897) / 2.0, np.arange(-64, 65) * 2.0 ** -11]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(B.e4m3(v), want)


@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (130, 129), (257, 300)])
def test_blocks_stand_for_their_values(group, rows, cols):
    rng = np.random.default_rng(rows + cols)
    x = rng.standard_normal((2, rows, cols)).astype(np.float32)
    q, s = B.quantize(x, group)
    assert q.shape == (2, rows, -(-cols // 128) * 128) and s.shape == (2, -(-cols // 128), -(-rows // group))
    got = B.dequantize(q, s, group)
    assert not got[:, :, cols:].any()
    # half a step of the value (2^-4 of it, or 2^-10 below the smallest normal value) and the three roundings of the scales
    bound = np.abs(x) * (2.0 ** -4 + 4 * 2.0 ** -24) + 2.0 ** -10 * np.repeat(np.repeat(s, group, 2)[:, :, :rows].transpose(0, 2, 1), 128, 2)[:, :, :cols]
    assert (np.abs(got[:, :, :cols] - x) <= bound).all()


def test_blocks_of_zeros_and_of_what_is_not_finite():
    x = np.zeros((1, 4, 256), np.float32)
    x[0, 1, 5], x[0, 2, 200], x[0, 3, 0] = np.nan, np.inf, 2.0 ** -140
    q, s = B.quantize(x, 1)
    assert s[0, 0, 0] == np.float32(2.0 ** -100) / np.float32(448) and not q[0, 0].any()
    assert np.isnan(s[0, 0, 1]) and np.isnan(q[0, 1, :128]).all() and s[0, 1, 1] == s[0, 0, 0]
    assert np.isposinf(s[0, 1, 2]) and np.isnan(B.dequantize(q, s, 1)[0, 2, 128:]).all()
    assert not q[0, 3].any()  # far below the smallest scale


def test_product_is_the_product_of_the_values():
    rng = np.random.default_rng(3)
    a, b = rng.standard_normal((2, 5, 200)).astype(np.float32), rng.standard_normal((2, 140, 200)).astype(np.float32)
    (qa, sa), (qb, sb) = B.quantize(a, 1), B.quantize(b, 128)
    got, size = B.product(qa, sa, qb, sb, 128)
    want = np.einsum("bmk,bnk->bmn", B.dequantize(qa, sa, 1), B.dequantize(qb, sb, 128))
    assert np.allclose(got, want, rtol=0, atol=1e-12) and (size >= np.abs(got) - 1e-12).all()


@pytest.mark.parametrize("kind,torch_act", [(B.ACT_NONE, lambda v: v), (B.ACT_RELU, torch.relu), (B.ACT_RELU6, torch.nn.functional.relu6),
                                            (B.ACT_GELU, torch.nn.functional.gelu), (B.ACT_SILU, torch.nn.functional.silu)])
def test_group_norm_is_torchs(kind, torch_act):
    rng = np.random.default_rng(4)
    x, gamma, beta = rng.standard_normal((2, 3, 5, 12)) * 3 + 1, rng.standard_normal(12), rng.standard_normal(12)
    got = B.group_norm(x, gamma, beta, 4, kind, 1e-3)[0]
    want = torch_act(torch.nn.functional.group_norm(torch.from_numpy(x).permute(0, 3, 1, 2), 4, torch.from_numpy(gamma), torch.from_numpy(beta), 1e-3))
    assert np.allclose(got, want.permute(0, 2, 3, 1).numpy(), rtol=1e-10, atol=1e-10)
