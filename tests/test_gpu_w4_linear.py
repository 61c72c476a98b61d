"""w4_linear against the product of the dequantized weights in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2101_05453_amd import binding  # noqa: E402


def make(M, K, N, group, seed=0):
    rng = np.random.default_rng(seed)
    codes = rng.integers(-8, 8, (N, K)).astype(np.int8)
    scales = (rng.standard_normal((N, -(-K // group))) * 0.01).astype(np.float32)
    x = rng.integers(-128, 128, (M, K)).astype(np.int8)
    return codes, scales, x, rng.uniform(0.001, 0.1, M).astype(np.float32), rng.standard_normal(N).astype(np.float32)


def check(y, codes, scales, group, x, a, zp=0, bias=None):
    """A group's sum is exact; its product with the scale, the sum over groups, the row's scale and the bias are float32:
    at most groups + 3 roundings of 2^-24 of what is summed, then one to y's type."""
    K = x.shape[1]
    w = codes.astype(np.float64) * np.repeat(scales.astype(np.float64), group, 1)[:, :K]
    xs = x.astype(np.float64) - zp
    a = np.broadcast_to(np.asarray(a, np.float32).astype(np.float64), x.shape[:1])[:, None]
    want = xs @ w.T * a
    terms = np.abs(xs) @ np.abs(w).T * a
    if bias is not None:
        want, terms = want + bias.astype(np.float64), terms + np.abs(bias)
    f = torch.finfo(y.dtype)
    bound = terms * (scales.shape[1] + 3) * 2.0 ** -24 + np.abs(want) * f.eps / 2 + f.smallest_normal * f.eps
    got = y.double().cpu().numpy()
    assert got.shape == want.shape and (np.abs(got - want) <= bound).all(), np.abs(got - want).max()


SIZES = [(1, 1, 1), (1, 128, 16), (1, 2048, 2048), (2, 75, 33), (3, 640, 1003), (7, 129, 17), (15, 1000, 100), (16, 256, 256), (17, 300, 65),
         (31, 96, 47), (33, 4096, 130), (64, 513, 200), (65, 128, 128), (100, 640, 77), (128, 384, 300), (129, 255, 129), (300, 200, 150),
         (513, 1024, 260), (1000, 640, 512),
         # enough rows and outputs for blocks of 128 x 128
         (33, 513, 16003), (65, 384, 8200), (129, 255, 5003), (300, 1000, 3001), (1000, 200, 1000), (2049, 130, 470), (17, 129, 14500)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M, K, N", SIZES)
def test_row_scales(M, K, N, group):
    codes, scales, x, a, bias = make(M, K, N, group, seed=M + K + N)
    m = binding.w4_prepare(codes=codes, scales=scales, group=group)
    mb = binding.w4_prepare(codes=codes, scales=scales, group=group, bias=bias)
    xd, ad = torch.from_numpy(x).cuda(), torch.from_numpy(a).cuda()
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        check(m.forward(xd, ad, dtype=dtype), codes, scales, group, x, a)
    check(mb.forward(xd, ad), codes, scales, group, x, a, bias=bias)
    check(mb.forward(xd, 0.25, zero_point=-128, dtype=torch.float32), codes, scales, group, x, 0.25, zp=-128, bias=bias)
    check(m.forward(xd, ad, zero_point=127, dtype=torch.float32), codes, scales, group, x, a, zp=127)


@pytest.mark.parametrize("M", [1, 40, 200])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_the_zero_point_is_exact(M, group):
    # rows of the zero point stand for zeros: nothing but the bias comes out
    codes, scales, _, _, bias = make(M, 333, 90, group)
    for zp in (-128, -1, 5, 127):
        x = torch.full((M, 333), zp, dtype=torch.int8, device="cuda")
        y = binding.w4_prepare(codes=codes, scales=scales, group=group, bias=bias).forward(x, 0.7, zero_point=zp, dtype=torch.float32)
        assert torch.equal(y.cpu(), torch.from_numpy(bias).expand(M, 90))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_blocks_of_a_zero_point_of_strided_rows_and_captured(group):
    M, K, N = 200, 333, 4003
    codes, scales, x, a, bias = make(M, K, N, group, seed=11)
    m = binding.w4_prepare(codes=codes, scales=scales, group=group, bias=bias)
    for zp in (-128, 127):
        y = m.forward(torch.full((M, K), zp, dtype=torch.int8, device="cuda"), 0.7, zero_point=zp, dtype=torch.float32)
        assert torch.equal(y.cpu(), torch.from_numpy(bias).expand(M, N))
    wide, out = torch.full((M, K + 9), 77, dtype=torch.int8, device="cuda"), torch.full((M, N + 5), -5.0, device="cuda")
    wide[:, 4:K + 4] = torch.from_numpy(x).cuda()
    ad, y = torch.from_numpy(a).cuda(), out[:, 2:N + 2]
    m.forward(wide[:, 4:K + 4], ad, y=y)
    check(y, codes, scales, group, x, a, bias=bias)
    assert (out[:, :2] == -5).all() and (out[:, N + 2:] == -5).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward(wide[:, 4:K + 4], ad, y=y)
    for k in range(3):
        x2 = np.roll(x, k + 1, 1)
        wide[:, 4:K + 4] = torch.from_numpy(x2).cuda()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(y, codes, scales, group, x2, a, bias=bias)


def test_quantized_here():
    rng = np.random.default_rng(4)
    W = rng.standard_normal((70, 200)).astype(np.float32)
    m = binding.w4_prepare(W=W, group=64)
    q = m.get_quant()
    x = rng.integers(-127, 128, (5, 200)).astype(np.int8)
    check(m.forward(torch.from_numpy(x).cuda(), 0.5, dtype=torch.float32), q["codes"], q["scales"], 64, x, 0.5)


@pytest.mark.parametrize("M", [5, 150])
def test_strided_rows_and_neighbours(M):
    codes, scales, x, a, _ = make(M, 203, 77, 64, seed=2)
    m = binding.w4_prepare(codes=codes, scales=scales, group=64)
    wide = torch.full((M, 301), 99, dtype=torch.int8, device="cuda")
    wide[:, 3:206] = torch.from_numpy(x).cuda()
    out = torch.full((M, 100), -5.0, device="cuda")
    y = m.forward(wide[:, 3:206], torch.from_numpy(a).cuda(), y=out[:, 11:88])
    check(y, codes, scales, 64, x, a)
    assert (out[:, :11] == -5).all() and (out[:, 88:] == -5).all()


@pytest.mark.parametrize("M, K", [(65536 * 64 + 5, 20), (65536 * 128 + 3, 130)])
def test_more_rows_than_a_grid_dimension_has(M, K):
    codes, scales, x, _, _ = make(997, K, 18, 32, seed=3)
    m = binding.w4_prepare(codes=codes, scales=scales, group=32)
    y = m.forward(torch.from_numpy(x).cuda().repeat(-(-M // 997), 1)[:M], 0.1)
    once = m.forward(torch.from_numpy(x).cuda(), 0.1)
    check(once, codes, scales, 32, x, 0.1)
    for at in (0, 997 * 500, M // 997 * 997 - 997):
        assert torch.equal(y[at:at + 997], once)
    assert torch.equal(y[M // 997 * 997:], once[:M % 997])


def test_leading_dimensions_an_empty_batch_and_refusals():
    codes, scales, x, a, _ = make(12, 64, 20, 32)
    m = binding.w4_prepare(codes=codes, scales=scales, group=32)
    xd, ad = torch.from_numpy(x).cuda(), torch.from_numpy(a).cuda()
    y = m.forward(xd.view(3, 4, 64), ad.view(3, 4))
    assert y.shape == (3, 4, 20) and torch.equal(y.view(12, 20), m.forward(xd, ad))
    assert m.forward(xd[:0], ad[:0]).shape == (0, 20)
    for bad in (lambda: m.forward(xd[:, :63], ad), lambda: m.forward(xd.float(), ad), lambda: m.forward(xd, ad[:3]), lambda: m.forward(xd, ad.double()),
                lambda: m.forward(xd.cpu(), 1.0), lambda: m.forward(xd, ad, y=torch.empty(12, 19, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(binding.LstmIntError):
        m.forward(xd, ad, zero_point=200)


def test_rows_of_unusable_scales_stay_by_themselves():
    codes, scales, x, a, _ = make(40, 96, 50, 32)
    a[7], a[9] = np.nan, np.inf
    y = binding.w4_prepare(codes=codes, scales=scales, group=32).forward(torch.from_numpy(x).cuda(), torch.from_numpy(a).cuda(), dtype=torch.float32)
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.isnan(y[7]).all() and not torch.isfinite(y[9]).any()
    check(y[keep], codes, scales, 32, x[keep], a[keep])


@pytest.mark.parametrize("M", [1, 48, 256])
def test_captured_and_on_another_stream(M):
    codes, scales, x, a, _ = make(M, 512, 384, 128, seed=6)
    m = binding.w4_prepare(codes=codes, scales=scales, group=128)
    xd, ad, y = torch.from_numpy(x).cuda(), torch.from_numpy(a).cuda(), torch.zeros(M, 384, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        m.forward(xd, ad, y=y)
    stream.synchronize()
    check(y, codes, scales, 128, x, a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward(xd, ad, y=y)
    for k in range(3):
        x2 = np.roll(x, k + 1, 1)
        xd.copy_(torch.from_numpy(x2))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(y, codes, scales, 128, x2, a)
        assert torch.equal(y, m.forward(xd, ad, dtype=torch.float32))


def test_more_than_a_launch_holds_is_refused():
    codes, scales, x, _, _ = make(64, 8, 1 << 17, 32)
    m = binding.w4_prepare(codes=codes, scales=scales, group=32)
    xd, y = torch.from_numpy(x).cuda(), torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    rc = binding.lm_lib()[0].w4_linear_forward(m._h, xd.data_ptr(), 8, 1 << 24, None, 1.0, 0, y.data_ptr(), 1 << 17, 2, None)
    torch.cuda.synchronize()
    assert rc == binding.E_UNSUPPORTED and not y.any()
