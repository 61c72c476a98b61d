"""rms_norm against its definition in 64 bits: codes equal, scales and floating outputs within their one rounding."""
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2101_05453_amd import binding  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6


def reference(x, weight, residual=None, gate=None, groups=1):
    r = x.double() + (residual.double() if residual is not None else 0)
    n = r.reshape(*r.shape[:-1], groups, -1)
    n = (n / torch.sqrt(n.pow(2).mean(-1, keepdim=True) + EPS) * weight.double()).reshape(r.shape)
    if gate is not None:
        n = n * gate.double() / (1 + torch.exp(-gate.double()))
    return r, n


def row_codes(n):
    most = n.abs().amax(-1, keepdim=True)
    return torch.where(most > 0, torch.floor(n / most * 127 + (0.5 + 2.0 ** -40)), torch.zeros_like(n)), most[..., 0] / 127


def make(rows, cols, dtype, groups=1, seed=0, lead=()):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x, res, gate = (draw(*lead, rows, cols).mul(torch.exp(draw(rows, 1))).to(dtype) for _ in range(3))
    return x, res, gate, torch.rand(cols // groups, generator=g) + 0.5


def near(got, want):
    """one rounding to got's type (two where it goes by way of float32: 2^-24 more), and its smallest step below the normal range"""
    f = torch.finfo(got.dtype)
    assert ((got.double().cpu() - want).abs() <= want.abs() * (f.eps / 2 + 2.0 ** -23) + f.smallest_normal * f.eps).all()


SIZES = [(1, 1, 1), (1, 2048, 1), (3, 7, 1), (2, 8, 1), (37, 1001, 1), (5, 2049, 1), (2, 8192, 1), (3, 8193, 1), (2, 32768, 1), (2, 32767, 1),
         (300, 512, 1), (4099, 64, 1), (5, 256, 2), (3, 4096, 32), (7, 12 * 75, 12), (2, 8 * 1000, 8), (1, 8192, 1024), (4, 9 * 9, 9),
         (3, 3 * 600, 3), (2, 4 * 2048, 4), (2, 2 * 1990, 2), (3, 15 * 513, 15), (1, 24, 3)]


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("rows, cols, groups", SIZES)
def test_codes_scales_and_outputs(rows, cols, groups, dtype):
    x, res, gate, w = make(rows, cols, dtype, groups, seed=rows + cols)
    for use_res, use_gate in ((False, False), (True, False), (False, True), (True, True)):
        r, n = reference(x, w, res if use_res else None, gate if use_gate else None, groups)
        xd, wd = x.cuda(), w.cuda()
        rd, gd = res.cuda() if use_res else None, gate.cuda() if use_gate else None
        y, new = torch.empty_like(xd), torch.empty_like(xd) if use_res else None
        codes, scales = binding.rms_norm_quantize(xd, wd, residual=rd, gate=gd, groups=groups, y=y, new_residual=new)
        want, s = row_codes(n)
        assert (codes.cpu().double() == want).all()
        near(scales, s)
        near(y, n)
        assert torch.equal(binding.rms_norm(xd, wd, residual=rd, gate=gd, groups=groups), y)
        if use_res:
            near(new, r)
        codes, none = binding.rms_norm_quantize(xd, wd, residual=rd, gate=gd, groups=groups, scale=0.031, zero_point=-7)
        assert none is None
        assert (codes.cpu().double() == (torch.floor(n / 0.031 + 0.5) - 7).clamp(-128, 127)).all()


def test_values_half_way_between_codes_go_up():
    # the row's largest is 127 eighths: odd sixteenths are half way
    x = torch.tensor([[127 / 8] + [k / 16 for k in range(-201, 202, 2)]], dtype=BF16)
    codes, _ = binding.rms_norm_quantize(x.cuda(), torch.ones(x.shape[1]).cuda())
    want = [(Fraction(float(v)) * 8 + Fraction(1, 2)).__floor__() for v in x[0]]
    assert codes[0].tolist() == want


def test_rows_without_a_scale():
    x = torch.randn(9, 700, generator=torch.Generator().manual_seed(3))
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 699] = float("inf")
    x[4] = float("-inf")
    x[5] = torch.finfo(FP32).max  # squares beyond float32
    x[6] = 2.0 ** -140  # subnormal
    codes, scales = binding.rms_norm_quantize(x.cuda(), torch.ones(700).cuda())
    codes, scales = codes.cpu(), scales.cpu()
    for row in (2, 3, 4):
        assert torch.isnan(scales[row]) and (codes[row] == 0).all()
    assert scales[1] == 0 and (codes[1] == 0).all()
    for row in (0, 5, 6, 7, 8):
        _, n = reference(x[row], torch.ones(700))
        want, s = row_codes(n)
        assert (codes[row].double() == want).all()
        near(scales[row:row + 1], s[None])
    static, _ = binding.rms_norm_quantize(x.cuda(), torch.ones(700).cuda(), scale=0.02, zero_point=4)
    assert (static[2] == 0).all() and static[3, 699] == 0 and (static[1] == 4).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_strided_rows_in_place_sum_and_neighbours(dtype):
    rows, cols = 11, 203
    x, res, _, w = make(rows, cols, dtype, seed=5)
    wide = torch.full((rows, 2 * cols + 3), 7.0, dtype=dtype)
    wide[:, 1:1 + cols], wide[:, 2 + cols:2 + 2 * cols] = x, res
    d = wide.cuda()
    xv, rv = d[:, 1:1 + cols], d[:, 2 + cols:2 + 2 * cols]
    r, n = reference(x, w, res)
    codes, scales = binding.rms_norm_quantize(xv, w.cuda(), residual=rv, new_residual=rv)
    assert (codes.cpu().double() == row_codes(n)[0]).all()
    near(rv, r)
    d = d.cpu()
    assert torch.equal(d[:, 1:1 + cols], x) and (d[:, 0] == 7).all() and (d[:, 1 + cols] == 7).all() and (d[:, 2 + 2 * cols:] == 7).all()


def test_leading_dimensions_and_an_empty_batch():
    x, _, _, w = make(6, 96, BF16, seed=8, lead=(4,))
    codes, scales = binding.rms_norm_quantize(x.cuda(), w.cuda())
    assert codes.shape == (4, 6, 96) and scales.shape == (4, 6)
    assert (codes.cpu().double() == row_codes(reference(x, w)[1])[0]).all()
    codes, scales = binding.rms_norm_quantize(x[:0].cuda(), w.cuda())
    assert codes.shape == (0, 6, 96) and scales.shape == (0, 6)
    with pytest.raises((ValueError, RuntimeError)):
        binding.rms_norm(x.cuda().transpose(1, 2), torch.ones(6).cuda())


def test_refusals_of_the_binding():
    x, w = torch.zeros(2, 64, dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    for bad in (lambda: binding.rms_norm(x, w[:63]), lambda: binding.rms_norm(x, w.half()), lambda: binding.rms_norm(x, w.cpu()),
                lambda: binding.rms_norm(x, w, residual=x[:1]), lambda: binding.rms_norm(x, w, gate=x.float()),
                lambda: binding.rms_norm_quantize(x, w, scale=0.0), lambda: binding.rms_norm_quantize(x, w, codes=x)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(binding.LstmIntError):
        binding.rms_norm(x, w, eps=-1.0)


def test_captured_and_on_another_stream():
    x, res, _, w = make(64, 640, BF16, seed=9)
    xd, rd, wd = x.cuda(), res.cuda(), w.cuda()
    codes, scales = torch.zeros(64, 640, dtype=torch.int8, device="cuda"), torch.zeros(64, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        binding.rms_norm_quantize(xd, wd, residual=rd, codes=codes, scales=scales)
    stream.synchronize()
    want = codes.clone(), scales.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.rms_norm_quantize(xd, wd, residual=rd, codes=codes, scales=scales)
    for k in range(3):
        xd.copy_(x.cuda() * 2.0 ** k)  # exact in any type
        rd.copy_(res.cuda() * 2.0 ** k)
        codes.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(codes, want[0])
        assert torch.allclose(scales, want[1], rtol=1e-5)  # eps beside a mean square that k changes
        assert np.isfinite(float((codes.float() * scales[:, None]).sum()))


# more threads than a dimension of a launch has (2^32), in rows of four waves and of a lane each
@pytest.mark.parametrize("rows, cols", [((1 << 24) + 5, 1025), ((1 << 29) + 999, 8)])
def test_more_rows_than_a_grid_dimension_has(rows, cols):
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    few, _, _, w = make(64, cols, BF16, seed=12)
    # behind the workgroups of the first dimension too: 2^21, of one row, and of 256
    spots = [0, (1 << 21) - 32, (1 << 23) - 32, rows - 64] if cols > 8 else [0, (1 << 29) - 32, rows - 64]
    for at in spots:
        x[at:at + 64] = few.cuda()
    codes, scales = binding.rms_norm_quantize(x, w.cuda())
    want, want_s = row_codes(reference(few, w)[1])
    for at in spots:
        assert (codes[at:at + 64].cpu().double() == want).all()
        near(scales[at:at + 64], want_s)
    assert int(torch.count_nonzero(scales)) == 64 * len(spots)
    del x, codes, scales
    torch.cuda.empty_cache()
