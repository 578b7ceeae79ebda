"""Products with weights in 4 bits at the ends of the range of x and of the zero points, in the kernels that take one or two vectors and in those of
the experts: sums of x that would leave the range of FP32 are formed element by element, and must be what the formula says all the same."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_w4 import U, Layer, Weights, call, check, close, rounded


def wide_zeros(w, rng):
    """zero points over the whole byte"""
    z = rng.integers(0, 256, w.z.shape).astype(np.uint8)
    at = np.arange(w.k) // w.group
    w.q = w.q + w.z[..., at].astype(np.float64) - z[..., at]
    w.w = w.s[..., at] * w.q
    w.size = np.abs(w.s[..., at]) * (32.0 + z[..., at])
    w.z = z
    w.gpu.zeros[..., :z.shape[-1]].copy_(torch.from_numpy(z))
    return w


def scaled(w, power):
    """the weights times 2^power"""
    w.gpu.scales.mul_(2.0 ** power)
    w.s, w.w, w.size = w.s * 2.0 ** power, w.w * 2.0 ** power, w.size * 2.0 ** power
    return w


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("t,k,group", [(1, 1024, 32), (2, 1500, 64), (1, 2050, 128), (2, 5000, 384), (1, 16383, 64), (4, 900, 32), (17, 1300, 128)])
def test_zero_points_of_a_whole_byte(x_type, t, k, group):
    rng = np.random.default_rng(k + t)
    print(x_type, t, k, group, flush=True)
    w = wide_zeros(Weights(rng, (), 45, k, group, True), rng)
    x, gx = rounded(rng.standard_normal((t, k)), x_type)
    close(oz.w4_matvec(w.gpu, gx, out=torch.empty((t, 45), device="cuda")), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("t,k,group", [(1, 1024, 64), (2, 1500, 64), (1, 2050, 32), (2, 2051, 128), (1, 16381, 1024), (2, 5000, 64)])
@pytest.mark.parametrize("zeros", [False, True])
def test_infinities_and_nans_follow_the_formula(x_type, t, k, group, zeros):
    rng = np.random.default_rng(k + t)
    n = 90
    print(x_type, t, k, group, zeros, flush=True)
    w = Weights(rng, (), n, k, group, zeros)
    x = rng.standard_normal((t, k))
    x[0, [70, k - 1]] = np.inf
    x[t - 1, 1000] = -np.inf if t > 1 else x[0, 1000]
    x, gx = rounded(x, x_type)
    got = oz.w4_matvec(w.gpu, gx, out=torch.empty((t, n), device="cuda")).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        sums = np.add.reduceat(w.q[None] * x[:, None, :], np.arange(0, k, group), axis=2)
        want = (sums * w.s[None]).sum(axis=2)
    assert np.isinf(want).any() and np.isnan(want).any()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    # a NaN in one vector alone: its results are NaN, the other's finite
    x, gx = rounded(rng.standard_normal((t, k)), x_type)
    gx[0, k - 2] = float("nan")
    got = oz.w4_matvec(w.gpu, gx, out=torch.empty((t, n), device="cuda"))
    assert bool(got[0].isnan().all())
    close(got[1:], x[1:] @ w.w.T, w.depth * U * (np.abs(x[1:]) @ w.size.T), "f32")


@pytest.mark.parametrize("t,k,group", [(1, 1024, 32), (2, 1500, 64), (1, 2050, 128), (2, 5001, 384), (1, 16384, 64)])
@pytest.mark.parametrize("x_type", ["f32", "bf16"])
def test_values_near_the_largest(x_type, t, k, group):
    """sums of x overflow, weights of 2^-20 of their size make finite results"""
    rng = np.random.default_rng(k)
    w = scaled(wide_zeros(Weights(rng, (), 37, k, group, True), rng), -20)
    x, gx = rounded(rng.standard_normal((t, k)) * 2.0 ** 122, x_type)
    close(oz.w4_matvec(w.gpu, gx, out=torch.empty((t, 37), device="cuda")), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")
    x = np.zeros((t, k))
    x[:, [3, k - 1]] = 3.3e38
    x, gx = rounded(x, x_type)
    close(oz.w4_matvec(w.gpu, gx, out=torch.empty((t, 37), device="cuda")), x @ w.w.T, w.depth * U * (np.abs(x) @ w.size.T), "f32")


@pytest.mark.parametrize("t,experts,top_k,d,f,group,zeros", [
    (1, 8, 3, 900, 700, 64, True), (1, 8, 3, 2100, 1500, 64, False), (4, 40, 3, 1000, 1001, 32, True), (4, 40, 3, 1100, 3001, 128, True),
    (3, 9, 3, 500, 777, 32, True), (3, 9, 3, 1030, 1300, 32, False), (12, 3, 2, 1030, 777, 64, True)])
def test_experts_with_tokens_and_inner_values_near_the_largest(t, experts, top_k, d, f, group, zeros):
    """tokens of about 2^116, gate's weights 2^-116, so that gate x is of ordinary size, up x as large as x, and h with it; down's are 2^-116"""
    rng = np.random.default_rng(d + t)
    print(t, experts, top_k, d, f, group, zeros, flush=True)
    layer = Layer(rng, experts, top_k, d, f, group, zeros=zeros, bias=list(rng.permutation(experts) * 0.1), score="sigmoid")
    layer.router = np.zeros_like(layer.router)
    layer.gpu.router.zero_()
    for part in (layer.gate, layer.down):
        scaled(part, -116)
    x, gx = rounded(rng.standard_normal((t, d)) * 2.0 ** 116, "f32")
    got = call(layer, gx)
    assert bool(got[0].isfinite().all())
    check(layer, x, got)
