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


HELD = 2.0 ** -25  # of the largest of a column and chunk: what two parts of fp16 leave of any of its numbers


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
