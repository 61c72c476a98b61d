"""rms_norm where its factors are far from one: codes are the definition's all the same."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2101_05453_amd import binding  # noqa: E402
from test_gpu_rms_norm import near, reference, row_codes  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def check(x, w, residual=None, gate=None, groups=1, scale=0.031, zero_point=-7):
    _, n = reference(x, w, residual, gate, groups)
    d = [None if t is None else t.cuda() for t in (x, w, residual, gate)]
    codes, scales = binding.rms_norm_quantize(d[0], d[1], residual=d[2], gate=d[3], groups=groups)
    want, s = row_codes(n)
    assert (codes.cpu().double() == want).all(), int((codes.cpu().double() != want).sum())
    near(scales, s)
    codes, _ = binding.rms_norm_quantize(d[0], d[1], residual=d[2], gate=d[3], groups=groups, scale=scale, zero_point=zero_point)
    want = (torch.floor(n / scale + 0.5) + zero_point).clamp(-128, 127)
    assert (codes.cpu().double() == want).all(), int((codes.cpu().double() != want).sum())


# products of two factors below float32's normal range, and a third that brings them back
@pytest.mark.parametrize("rows, cols", [(3, 500), (2, 3000), (1, 20000)])
def test_columns_whose_weight_is_as_large_as_their_values_are_small(rows, cols):
    g = torch.Generator().manual_seed(cols)
    x, w = torch.randn(rows, cols, generator=g), torch.rand(cols, generator=g) + 0.5
    w = w * 2.0 ** -14
    x[:, ::3] *= 2.0 ** -141
    w[::3] *= 2.0 ** 70  # twice: a factor of 2^140 is infinite in float32
    w[::3] *= 2.0 ** 70
    assert torch.isfinite(w).all()
    check(x, w, scale=2.0 ** -20)


@pytest.mark.parametrize("groups", [1, 5])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gates_as_large_as_weights_are_small(groups, dtype):
    g = torch.Generator().manual_seed(groups)
    x, gate = (torch.randn(4, 700, generator=g) for _ in range(2))
    w = torch.rand(700 // groups, generator=g) + 0.5
    x[:, ::6] *= 2.0 ** -60  # times their weights 2^-140
    w = torch.where(torch.arange(700 // groups) % 2 == 0, w * 2.0 ** -80, w * 2.0 ** -10)
    gate[:, ::6] = gate[:, ::6].abs() * 2.0 ** 126
    check(x.to(dtype), w, gate=gate.to(dtype), groups=groups, scale=2.0 ** -18)


# a gate of -90: its factor is below float32's normal range, the weight brings it back
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_weights_as_large_as_gates_factors_are_small(dtype):
    g = torch.Generator().manual_seed(5)
    x, gate = (torch.randn(4, 700, generator=g) for _ in range(2))
    w = torch.rand(700, generator=g) + 0.5
    gate[:, ::7] = -torch.linspace(80, 104, 100)
    w[::7] *= 2.0 ** 120
    check(x.to(dtype), w, gate=gate.to(dtype), scale=0.0311)


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_gates_that_are_closed(groups, dtype):
    g = torch.Generator().manual_seed(6)
    x, gate = (torch.randn(5, 1024, generator=g) for _ in range(2))
    for i, z in enumerate((-80.0, -87.5, -88.5, -89.0, -200.0, -1e4, 80.0, 1e4)):
        gate[:, 10 + 100 * i] = z
    gate[4] = -1e4  # a row of nothing but closed gates: codes 0
    check(x.to(dtype), torch.rand(1024 // groups, generator=g) + 0.5, gate=gate.to(dtype), groups=groups)


def test_a_zero_point_without_a_scale_is_refused():
    x, w = torch.ones(2, 64, dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    with pytest.raises(AssertionError):
        binding.rms_norm_quantize(x, w, zero_point=5)
    codes, _ = binding.rms_norm_quantize(x, w, scale=1.0, zero_point=5)
    assert (codes == 6).all()
