"""The norm of rows of any size: elements from the least to the largest of bf16, whose squares fp32 does not hold.

    |out - ref| <= 2^-8 |ref| + 2^-18 (|y_j| + |y_(j + d/2)|) + 2^-133
as in test_gpu_tree.py (the norm takes as many roundings at any size: the scaling by powers of two is exact, except that 1 / root has 2^-22
where it is below 2^-126); below 2^-126 a rounding to bf16 is off by 2^-134, those to fp32 by 2^-150, a dozen of them."""
import numpy as np
import pytest
import torch

import tree_reference as ref

pytestmark = pytest.mark.gpu

cm = pytest.importorskip("paper_2607_01308_gb300")

DEV = "cuda:0"
THETA = 1.0e6


@pytest.fixture(scope="module")
def ctx():
    c = cm.Context(0, rope_theta=THETA)
    yield c
    c.close()


def _check(x, got, positions, weight, eps):
    want, size = ref.rotate(x.double().numpy(), positions.numpy(), weight.double().numpy(), float(np.float32(eps)), THETA)
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size + 2.0 ** -133), np.nanmax(err / (np.abs(want) + 2.0 ** -133))


def _rows(rows, heads, d, seed):
    """Rows of every size, in any order, some constant, some with one element that is larger or smaller than the others by far."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, heads, d), generator=g, dtype=torch.float64).clamp(-5, 5)
    power = torch.randint(-133, 126, (rows, heads, 1), generator=g).double()
    x[::5] = torch.sign(x[::5])
    x = x * torch.exp2(power)
    at = torch.randint(0, d, (rows,), generator=g)
    every = torch.arange(rows)
    x[every[1::7], 0, at[1::7]] = 2.0 ** 126
    x[every[2::7], 0, at[2::7]] = 2.0 ** -130
    x[3::11, heads - 1] = 0
    return x.bfloat16()


@pytest.mark.parametrize("d", [16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-30, 1e-18, 1e-6, 3e38])
def test_rotate_rows_of_any_size(ctx, d, eps):
    x = _rows(301, 4, d, d)
    w = torch.randn(d, generator=torch.Generator().manual_seed(1)).bfloat16()
    pos = torch.randint(-5, 100000, (301,), generator=torch.Generator().manual_seed(2)).int()
    gpu = x.to(DEV)
    q, k = cm.rotate_qk(ctx, gpu[:, :3], gpu[:, 3:], pos.to(DEV), w.to(DEV), w.to(DEV), eps=eps)
    _check(x[:, :3], q, pos, w, eps)
    _check(x[:, 3:], k, pos, w, eps)


def test_rotate_small_rows_without_eps(ctx):
    """x / sqrt(mean x^2) is of size 1 whatever x is."""
    for size in (2.0 ** -133, 1e-30, 1e-23, 1e-19, 1e-12, 1e18, 1e30, 3.3895e38):
        x = torch.full((3, 2, 32), size, dtype=torch.float64).bfloat16()
        q, _ = cm.rotate_qk(ctx, x.to(DEV), None, _i32_zeros(3), torch.ones(32, dtype=torch.bfloat16, device=DEV), eps=0.0)
        assert bool((q == 1).all())


def _i32_zeros(n):
    return torch.zeros(n, dtype=torch.int32, device=DEV)


def test_rotate_one_norm_alone_leaves_the_other(ctx):
    """Rows without a weight are not normed, however large or small they are."""
    x = _rows(64, 4, 64, 9)
    gpu, w = x.to(DEV), torch.ones(64, dtype=torch.bfloat16, device=DEV)
    q, k = cm.rotate_qk(ctx, gpu[:, :2], gpu[:, 2:], _i32_zeros(64), w, None, eps=0.0)
    assert torch.equal(k, gpu[:, 2:])
    _check(x[:, :2], q, torch.zeros(64).int(), torch.ones(64), 0.0)
