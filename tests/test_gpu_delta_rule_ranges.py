"""delta_rule where the state, the decays and the values leave the ordinary range: bounds that forget as the state does."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2101_05453_amd import binding  # noqa: E402

BF16, FP32 = torch.bfloat16, torch.float32
# B, Hk, Hv, Dk, Dv: few heads; columns that no tile divides; 256 key columns; enough heads for 128 columns to a workgroup
SIZES = [(1, 1, 2, 64, 48), (2, 1, 1, 128, 75), (1, 1, 1, 200, 32), (70, 2, 4, 64, 100)]


def make(T, B, Hk, Hv, Dk, Dv, dtype, seed):
    n = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(T, B, h, d, generator=n).to(dtype) for h, d in ((Hk, Dk), (Hk, Dk), (Hv, Dv)))
    g = -0.5 * torch.rand(T, B, Hv, generator=n)
    beta = torch.sigmoid(torch.randn(T, B, Hv, generator=n))
    return [q, k, v, g, beta, torch.randn(B, Hv, Dk, Dv, generator=n) / math.sqrt(Dk)]


def reference(q, k, v, g, beta, S):
    """The recurrence in 64 bits: y, the state, and for each step and head what a rounding is a part of: the first state's norm
    and those of all writes, decayed as the state is."""
    q, k, v, g, beta, S = (t.double().numpy() for t in (q, k, v, g, beta, S))
    q, k = (np.repeat(t / np.sqrt((t * t).sum(3, keepdims=True) + 1e-6), v.shape[2] // k.shape[2], 2) for t in (q, k))
    norm = lambda x, axes: np.sqrt((x * x).sum(axes))  # noqa: E731
    q, size = q * k.shape[3] ** -0.5, norm(S, (2, 3))
    y, sizes = np.zeros(v.shape), np.zeros(g.shape)
    for t in range(len(v)):
        e = np.exp(g[t])
        S = S * e[:, :, None, None]
        Sk = (S * k[t][..., None]).sum(2)
        u = beta[t][..., None] * (v[t] - Sk)
        S = S + k[t][..., None] * u[:, :, None]
        size = size * e + beta[t] * (norm(v[t], 2) + norm(Sk, 2))
        y[t], sizes[t] = (S * q[t][..., None]).sum(2), size
    return y, S, sizes


HELD = 2.0 ** -39  # of the largest of a column and chunk: what two parts of fp16 leave of any of its numbers


def check(args, y, state, scale_q):
    """A step contracts the state and its error alike (|k| <= 1, 0 <= beta <= 1) and adds the roundings of a few sums over Dk:
    (8 + sqrt(Dk)) of 2^-24 of the decayed sizes, like a random walk over the steps, 4 as its margin.  What a chunk of 32 steps holds
    in two parts of fp16 is off by HELD of the largest that it holds in a column, however small it is by itself: at four
    places, each a sum over 32 steps, 128 HELD of the chunk's largest size.  That error is in the state from there on, and
    decays as it does.  Numbers below 2^-100 have no bound of their own."""
    want_y, want_S, sizes = reference(*args)
    T, Dk = len(want_y), want_S.shape[2]
    decay = np.exp(args[3].double().numpy())
    held, carried = np.zeros_like(sizes), np.zeros_like(sizes[0])
    for t in range(T):
        if t % 32 == 0:
            new = 128 * HELD * sizes[t:t + 32].max(0)
        carried = carried * decay[t]
        held[t] = new + carried
        if t % 32 == 31:
            carried = held[t]
    bound = 4 * math.sqrt(T + 1) * (8 + math.sqrt(Dk)) * 2.0 ** -24 * sizes + held + 2.0 ** -100
    y, state = y.double().cpu().numpy(), state.double().cpu().numpy()
    assert np.isfinite(y).all() and np.isfinite(state).all()
    off = np.sqrt(((state - want_S) ** 2).sum((2, 3)))
    assert (off <= bound[-1]).all(), (off / bound[-1]).max()
    f = torch.finfo(args[2].dtype)
    off = np.sqrt((np.maximum(np.abs(y - want_y) - np.abs(want_y) * f.eps / 2, 0) ** 2).sum(3))
    assert (off <= bound * scale_q + f.smallest_normal * f.eps * 16).all(), (off / bound / scale_q).max()


def run_and_check(args):
    d = [t.cuda() for t in args]
    y = binding.delta_rule(*d[:5], state=d[5], normalize=True)
    check(args, y, d[5], args[1].shape[3] ** -0.5)


# 96 steps in which the state fades and nothing is written, decays of 84 to 103 a chunk, then ordinary steps
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("nothing", ["beta", "v"])
@pytest.mark.parametrize("size, decay", [(1e4, 2.7), (3e5, 2.95), (1e6, 2.65), (1e6, 2.95), (1e7, 3.2)])
@pytest.mark.parametrize("B, Hk, Hv, Dk, Dv", SIZES)
def test_a_large_state_that_fades(B, Hk, Hv, Dk, Dv, size, decay, nothing, dtype):
    args = make(140, B, Hk, Hv, Dk, Dv, dtype, seed=Dk)
    args[5] *= size
    args[3][:96] = -decay
    args[4 if nothing == "beta" else 2][:96] = 0
    run_and_check(args)


# a state that has faded below what its scale reaches, and then a loud value
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("loud", [1.0, 3e3, 1e5, 1e30])
@pytest.mark.parametrize("B, Hk, Hv, Dk, Dv", SIZES)
def test_loud_values_after_a_state_that_has_faded(B, Hk, Hv, Dk, Dv, loud, dtype):
    args = make(330, B, Hk, Hv, Dk, Dv, dtype, seed=Dk + 1)
    args[2][:290] = 0
    args[2][290:] *= loud
    args[3][:290] = -0.5
    run_and_check(args)


# one step forgets, the steps after it write nothing until the next chunk begins
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("at", [0, 20, 31])
@pytest.mark.parametrize("decay", [60.0, 85.0, 95.0, 103.0, 200.0])
def test_a_step_that_forgets_and_none_that_write(decay, at, dtype):
    args = make(100, 1, 1, 2, 64, 48, dtype, seed=5)
    args[5] *= 1e4
    args[3][32 + at] = -decay
    args[4][32 + at:64] = 0
    run_and_check(args)


# whole columns of nothing, then values of any size
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_columns_that_begin_at_nothing(dtype):
    args = make(100, 1, 1, 2, 64, 48, dtype, seed=6)
    args[5].zero_()
    args[2][:64] = 0
    args[2][64:, :, 0] *= 1e25
    args[2][64:, :, 1] *= 1e-25
    run_and_check(args)


# a column whose scale is that of a large state, which is cleared, and then gets something far smaller
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", [1e10, 1e33])
def test_a_cleared_state_and_small_values(size, dtype):
    args = make(100, 1, 1, 2, 64, 48, dtype, seed=7)
    args[5] *= size
    args[2] *= 1e-20
    args[3][32] = float("-inf")
    run_and_check(args)


# A value far louder than the others, at the last step of a chunk: the outputs before it are of the size they have without it.
# Per column: the roundings of check(), and 2^-39 of the chunk's largest value, at two places (the right-hand side, u) and in
# a sum over 32 steps of products of unit vectors.
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("loud", [1e3, 1e5, 1e7])
@pytest.mark.parametrize("B, Hk, Hv, Dk, Dv", SIZES)
def test_a_loud_step_leaves_the_steps_before_it(B, Hk, Hv, Dk, Dv, loud, dtype):
    T = 64
    args = make(T, B, Hk, Hv, Dk, Dv, dtype, seed=Dk + 2)
    want = reference(*args)[0]
    args[2][63] *= loud
    d = [t.cuda() for t in args]
    y = binding.delta_rule(*d[:5], state=d[5], normalize=True).double().cpu().numpy()[:63]
    quiet = [t[:63] for t in args[:5]] + [args[5]]
    sizes = reference(*quiet)[2]
    walk = 4 * math.sqrt(T + 1) * (8 + math.sqrt(Dk)) * 2.0 ** -24 * sizes[..., None]
    largest = np.abs(args[2].double().numpy()).max(0)
    off = np.abs(y - want[:63]) - np.abs(want[:63]) * torch.finfo(dtype).eps / 2
    bound = (walk + 64 * 2.0 ** -39 * largest) * Dk ** -0.5
    assert (off <= bound).all(), (off / bound).max()
    assert loud > 1e5 or (off <= 1e-3 * np.sqrt((want[:63] ** 2).mean())).all()


# A value far louder than the others, forgotten within its chunk: what comes behind it is of its own size.  Per column, as above:
# what is off is 2^-39 of the loud value, not of what is left of it.
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("loud", [1e3, 1e5, 1e7])
@pytest.mark.parametrize("at", [5, 30])
def test_a_loud_value_is_forgotten(at, loud, dtype):
    args = make(64, 1, 1, 2, 64, 48, dtype, seed=8)
    args[2][at] *= loud
    args[3][at + 1] = -math.log(loud) - 6
    run_and_check(args)


# Float32 outputs, step by step: a sum of Dk or 32 products, each off by 2^-22 of itself and independent of the others, is off by
# 2^-22 of the root of the sum of their squares: for a query of normal draws |S| / sqrt(Dk), with |S| the root of the squares
# of the first state and all writes, decayed.  A chunk's seven products add theirs to the state, and chunks add up like a
# random walk.  16 for the seven products, for sums in float32 and for the largest of many draws; leaving out one low part of
# any operand is 500 and more.
@pytest.mark.parametrize("T, B, Hk, Hv, Dk, Dv", [(16, 1, 1, 1, 128, 128), (33, 2, 1, 2, 100, 50), (64, 1, 1, 1, 128, 128), (130, 1, 1, 2, 256, 64),
                                                  (200, 3, 2, 2, 128, 128), (257, 1, 1, 1, 200, 256), (300, 1, 3, 6, 16, 48), (500, 1, 1, 1, 7, 5),
                                                  (70, 70, 2, 4, 128, 100)])
def test_every_output_has_the_bits_of_float32(T, B, Hk, Hv, Dk, Dv):
    args = make(T, B, Hk, Hv, Dk, Dv, FP32, seed=T)
    want, want_S, _ = reference(*args)
    d = [t.cuda() for t in args]
    y = binding.delta_rule(*d[:5], state=d[5], normalize=True).double().cpu().numpy()
    k, v, g, beta, S = (t.double().numpy() for t in args[1:])
    k = np.repeat(k / np.sqrt((k * k).sum(3, keepdims=True) + 1e-6), Hv // Hk, 2)
    n2 = (S * S).sum((2, 3))
    for t in range(T):
        S = S * np.exp(g[t])[:, :, None, None]
        Sk = (S * k[t][..., None]).sum(2)
        n2 = n2 * np.exp(2 * g[t]) + beta[t] ** 2 * ((v[t] ** 2).sum(2) + (Sk ** 2).sum(2))
        S = S + k[t][..., None] * (beta[t][..., None] * (v[t] - Sk))[:, :, None]
        bound = 16 * 2.0 ** -22 * np.sqrt(n2 / Dk * (1 + t / 32)) * Dk ** -0.5
        off = np.sqrt(((y[t] - want[t]) ** 2).sum(2))
        assert (off <= bound).all(), (t, (off / bound).max())
    off = np.sqrt(((d[5].double().cpu().numpy() - want_S) ** 2).sum((2, 3)))
    assert (off <= 16 * 2.0 ** -22 * np.sqrt(n2 * (1 + T / 32))).all()
