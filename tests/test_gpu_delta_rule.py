"""delta_rule against the recurrence in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2101_05453_amd import binding  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def make(T, B, Hk, Hv, Dk, Dv, dtype, normalize=True, seed=0, slow=False, alike=False):
    """slow: hardly any decay.  alike: keys that point nearly the same way, as neighbouring tokens' do."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    q, k, v = n(T, B, Hk, Dk), n(T, B, Hk, Dk), n(T, B, Hv, Dv)
    if alike:
        k = n(1, 1, Hk, Dk) + 0.1 * k
    if not normalize:
        q, k = (t / t.norm(dim=3, keepdim=True).clamp_min(1e-9) for t in (q, k))
    decay = -torch.exp(torch.rand(1, 1, Hv, generator=g) * 7 - 6.5) * (torch.rand(T, B, Hv, generator=g) + 0.1)
    if slow:
        decay = decay * 1e-4
    beta = torch.ones(T, B, Hv) if alike else torch.sigmoid(n(T, B, Hv))
    return q.to(dtype), k.to(dtype), v.to(dtype), decay, beta, n(B, Hv, Dk, Dv) / math.sqrt(Dk)


def reference(q, k, v, g, beta, state=None, lengths=None, normalize=True, scale=None):
    q, k, v, g, beta = (t.double().cpu().numpy() for t in (q, k, v, g, beta))
    T, B, Hv, Dv = v.shape
    Hk, Dk = k.shape[2:]
    S = np.zeros((B, Hv, Dk, Dv)) if state is None else state.double().cpu().numpy().copy()
    y = np.zeros(v.shape)
    if normalize:
        q, k = (t / np.sqrt((t * t).sum(3, keepdims=True) + 1e-6) for t in (q, k))
    q, k = (np.repeat(t, Hv // Hk, 2) for t in (q * (Dk ** -0.5 if scale is None else scale), k))
    most = 1.0  # the largest norm that a head's state or value had
    for t in range(T):
        with np.errstate(over="ignore"):
            new = S * np.exp(g[t])[:, :, None, None]
        u = beta[t][:, :, None] * (v[t] - np.einsum("bhkv,bhk->bhv", new, k[t]))
        new = new + k[t][..., None] * u[:, :, None]
        live = np.ones((B, 1, 1, 1), bool) if lengths is None else (lengths.cpu().numpy() > t)[:, None, None, None]
        S = np.where(live, new, S)
        y[t] = np.einsum("bhkv,bhk->bhv", S, q[t]) * live[..., 0]
        most = max(most, np.sqrt((S * S).sum((2, 3))).max(initial=0), np.abs(v[t]).max(initial=0) * math.sqrt(Dv))
    return y, S, most


def check(got, state, want, T, scale_q):
    """The step is a contraction of the state where |k| <= 1 and 0 <= beta <= 1, so the rounding of each step adds up: like
    a random walk, sqrt(T + 1) steps, each of a few sums over Dk, (8 + sqrt(Dk)) roundings of 2^-24 of the largest norm, with
    4 as the margin of a walk.  An output is that times its query, and one rounding to its type."""
    y, S, most = want
    Dk = S.shape[2]
    walk = 4 * math.sqrt(T + 1) * (8 + math.sqrt(Dk)) * 2.0 ** -24 * most
    if state is not None:
        off = state.double().cpu().numpy() - S
        assert np.sqrt((off * off).sum((2, 3))).max(initial=0) <= walk, (np.sqrt((off * off).sum((2, 3))).max(), walk)
    f = torch.finfo(got.dtype)
    off = np.abs(got.double().cpu().numpy() - y)
    bound = walk * scale_q + np.abs(y) * f.eps / 2 + f.smallest_normal * f.eps
    assert (off <= bound).all(), (off.max(), (off - bound).max())


def run(args, normalize=True, **kw):
    q, k, v, g, beta, state = (t.cuda() for t in args)
    y = binding.delta_rule(q, k, v, g, beta, state=state, normalize=normalize, **kw)
    return y, state


SIZES = [(1, 1, 1, 1, 128, 128), (1, 3, 2, 4, 64, 64), (1, 2, 1, 1, 1, 1), (2, 1, 1, 3, 17, 33), (5, 2, 2, 2, 128, 80), (15, 1, 1, 2, 96, 16),
         (16, 1, 1, 1, 128, 128), (33, 2, 1, 2, 100, 50), (63, 1, 2, 2, 64, 64), (64, 1, 1, 1, 128, 128), (65, 2, 1, 2, 128, 96),
         (127, 1, 1, 1, 75, 130), (128, 2, 2, 4, 32, 17), (130, 1, 1, 2, 256, 64), (200, 3, 2, 2, 128, 128), (257, 1, 1, 1, 200, 256),
         (300, 1, 3, 6, 16, 48), (500, 1, 1, 1, 7, 5),
         # single steps of many heads; many chunks whose value heads share a key head
         (1, 130, 4, 8, 128, 40), (3, 70, 2, 16, 33, 50), (70, 350, 4, 12, 32, 16), (130, 211, 4, 4, 20, 12)]


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("T, B, Hk, Hv, Dk, Dv", SIZES)
def test_sequences(T, B, Hk, Hv, Dk, Dv, dtype):
    args = make(T, B, Hk, Hv, Dk, Dv, dtype, seed=T + Dk)
    y, state = run(args)
    check(y, state, reference(*args), T, Dk ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("T", [1, 3, 64, 190])
def test_unit_keys_without_normalizing_and_an_own_scale(T, dtype):
    args = make(T, 2, 2, 2, 96, 64, dtype, normalize=False, seed=T)
    y, state = run(args, normalize=False, scale=0.7)
    # a key rounded to its type is up to 2^-8 longer than one: the step may grow by that, over T steps by a factor of two
    check(y, state, reference(*args, normalize=False, scale=0.7), 4 * T, 0.7 * 2)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("alike", [False, True])
def test_slow_decay_and_keys_that_are_alike(dtype, alike):
    args = make(400, 1, 2, 4, 128, 64, dtype, seed=3, slow=True, alike=alike)
    y, state = run(args)
    check(y, state, reference(*args), 400, 128 ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("T", [3, 150])
def test_lengths(T, dtype):
    B = 6
    q, k, v, g, beta, state = make(T, B, 1, 2, 64, 48, dtype, seed=5)
    lengths = torch.tensor([T, 0, 1, T - 1, T // 2, 2], dtype=torch.int32)
    want = reference(q, k, v, g, beta, state, lengths)
    for b in range(B):  # nothing behind a row's end is looked at
        for t in (q, k, v, g, beta):
            t[lengths[b]:, b] = float("nan")
    y = torch.full(v.shape, 3.0, dtype=dtype, device="cuda")
    new = torch.full_like(state, 9.0).cuda()
    args = [t.cuda() for t in (q, k, v, g, beta)]
    binding.delta_rule(*args, state=state.cuda(), new_state=new, lengths=lengths.cuda(), normalize=True, y=y)
    for b in range(B):
        assert (y[lengths[b]:, b] == 3).all()
        y[lengths[b]:, b] = 0
    check(y, new, want, T, 64 ** -0.5)
    assert torch.equal(new[1].cpu(), state[1])
    # lengths out of range are brought into it
    wild = torch.tensor([T + 100, -5, 1, T - 1, T // 2, 2], dtype=torch.int32).cuda()
    y2 = binding.delta_rule(*args, state=state.cuda(), lengths=wild, normalize=True)
    assert torch.equal(y2, y)


@pytest.mark.parametrize("T", [1, 100])
def test_states_given_kept_and_left_out(T):
    args = make(T, 2, 1, 2, 64, 64, BF16, seed=6)
    state = args[-1]
    d = [t.cuda() for t in args]
    new = torch.empty_like(d[-1])
    y = binding.delta_rule(*d[:5], state=d[5], new_state=new, normalize=True)
    assert torch.equal(d[5].cpu(), state)
    in_place = d[5].clone()
    y2 = binding.delta_rule(*d[:5], state=in_place, normalize=True)
    assert torch.equal(y, y2) and torch.equal(in_place, new)
    zeros = binding.delta_rule(*d[:5], new_state=new, normalize=True)
    check(zeros, new, reference(*args[:5]), T, 64 ** -0.5)
    assert torch.equal(zeros, binding.delta_rule(*d[:5], normalize=True))
    assert torch.equal(zeros, binding.delta_rule(*d[:5], state=torch.zeros_like(new), normalize=True))


def test_no_steps_copies_the_state():
    args = [t.cuda() for t in make(0, 2, 1, 2, 64, 20, BF16)]
    new = torch.full_like(args[5], 5.0)
    y = binding.delta_rule(*args[:5], state=args[5], new_state=new)
    assert y.shape == (0, 2, 2, 20) and torch.equal(new, args[5])
    binding.delta_rule(*args[:5], new_state=new)
    assert (new == 0).all()


def test_a_long_sequence_in_pieces():
    T = 330
    args = make(T, 2, 2, 4, 128, 64, BF16, seed=7)
    want = reference(*args)
    d = [t.cuda() for t in args]
    ys, at = [], 0
    for n in (1, 64, 3, 200, 1, 61):
        ys.append(binding.delta_rule(*(t[at:at + n] for t in d[:5]), state=d[5], normalize=True))
        at += n
    assert at == T
    check(torch.cat(ys), d[5], want, T, 128 ** -0.5)


@pytest.mark.parametrize("T", [2, 70])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_strides(T, dtype):
    B, Hk, Hv, Dk, Dv = 3, 2, 4, 72, 40
    args = make(T, B, Hk, Hv, Dk, Dv, dtype, seed=8)
    q, k, v, g, beta, state = args
    # q, k and v side by side in rows of odd length; g and beta with the heads first; y with the batch first
    width = 2 * Hk * Dk + Hv * Dv + 1
    qkv = torch.full((T, B, width), 50.0, dtype=dtype)
    qkv[..., :Hk * Dk], qkv[..., Hk * Dk:2 * Hk * Dk], qkv[..., 2 * Hk * Dk:-1] = q.flatten(2), k.flatten(2), v.flatten(2)
    qkv = qkv.cuda()
    qd, kd = (qkv[..., i * Hk * Dk:(i + 1) * Hk * Dk].unflatten(2, (Hk, Dk)) for i in (0, 1))
    vd = qkv[..., 2 * Hk * Dk:-1].unflatten(2, (Hv, Dv))
    gd, bd = (t.permute(2, 1, 0).contiguous().permute(2, 1, 0) for t in (g.cuda(), beta.cuda()))
    room = torch.full((B, T, Hv, Dv + 3), 8.0, dtype=dtype, device="cuda")
    y = room[..., 1:Dv + 1].transpose(0, 1)
    sd = state.cuda()
    binding.delta_rule(qd, kd, vd, gd, bd, state=sd, normalize=True, y=y)
    check(y, sd, reference(*args), T, Dk ** -0.5)
    assert (room[..., 0] == 8).all() and (room[..., Dv + 1:] == 8).all()
    # one set of heads for the whole batch, by a stride of zero
    one = [t[:, :1].cuda().expand(-1, B, *t.shape[2:]) for t in (q, k, v, g, beta)]
    sd = state.cuda()
    y = binding.delta_rule(*one, state=sd, normalize=True)
    check(y, sd, reference(*(t.contiguous() for t in one), state), T, Dk ** -0.5)


@pytest.mark.parametrize("T", [4, 150])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_decays_of_nothing_and_rates_of_nothing(T, dtype):
    q, k, v, g, beta, state = make(T, 1, 1, 3, 64, 32, dtype, seed=9)
    g[T // 2:T // 2 + 2, :, 0] = float("-inf")  # the state is cleared
    g[:, :, 1] = 0  # no decay
    g[T // 2:, :, 2] = -200.0  # a decay below float32's range
    beta[:, :, 1] = 0  # nothing is written
    y, new = run((q, k, v, g, beta, state))
    check(y, new, reference(q, k, v, g, beta, state), T, 64 ** -0.5)
    assert torch.equal(new[0, 1].cpu(), state[0, 1])


def test_sums_of_decay_are_taken_where_they_matter():
    # a step of a large decay within a chunk: what comes after it still has its own, small ones
    q, k, v, g, beta, state = make(64, 1, 1, 1, 64, 64, FP32, seed=10, slow=True)
    g[20] = -900.0
    g[40] = float("-inf")
    y, new = run((q, k, v, g, beta, state))
    check(y, new, reference(q, k, v, g, beta, state), 64, 64 ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("by", [1e-25, 1e-6, 1e6, 1e25])
def test_magnitudes(by, dtype):
    # states and values far from one, columns far from each other, and a state far from what is written to it
    q, k, v, g, beta, state = make(100, 1, 1, 2, 64, 48, dtype, seed=13)
    columns = 10.0 ** torch.linspace(-5, 5, 48)
    v, state = (v.float() * by * columns).to(dtype), state * by * columns
    state[:, 1] *= 1e-6
    y, new = run((q, k, v, g, beta, state))
    want = reference(q, k, v, g, beta, state)
    for c in range(48):  # the bound of check(), for each column by itself
        s = float(columns[c]) * by
        part = [want[0][..., c:c + 1] / s, want[1][..., c:c + 1] / s]
        most = max(1.0, np.sqrt((part[1] ** 2).sum((2, 3))).max(), float((v[..., c].double() / s).abs().max()), float(state[..., c].norm(dim=2).max() / s))
        walk = 4 * 101 ** 0.5 * 16 * 2.0 ** -24 * most
        assert np.abs(new[..., c].double().cpu().numpy() / s - part[1][..., 0]).max() <= walk
        off = np.abs(y[..., c].double().cpu().numpy() / s - part[0][..., 0])
        f = torch.finfo(dtype)
        assert (off <= walk * 64 ** -0.5 + np.abs(part[0][..., 0]) * f.eps / 2 + f.smallest_normal * f.eps / s).all()


def test_values_that_are_not_finite_stay_in_their_head_and_row():
    T = 100
    args = make(T, 2, 2, 2, 64, 32, BF16, seed=11)
    want = reference(*args)
    v = args[2].clone()
    v[70, 0, 1, 3] = float("nan")
    y, state = run((args[0], args[1], v, *args[3:]))
    assert torch.isnan(y[70:, 0, 1, 3]).all() and torch.isnan(state[0, 1, :, 3]).all()
    y[:, 0, 1], state[0, 1] = 0, 0
    want[0][:, 0, 1], want[1][0, 1] = 0, 0
    check(y, state, want, T, 64 ** -0.5)


# many chunks, whose value heads share what is made of a key head
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_heads_that_share_keys_with_lengths_and_values_that_are_not_finite(dtype):
    T, B, Hk, Hv = 70, 350, 4, 12
    args = make(T, B, Hk, Hv, 40, 24, dtype, seed=13)
    lengths = torch.randint(0, T + 1, (B,), generator=torch.Generator().manual_seed(14), dtype=torch.int32)
    lengths[:6] = torch.tensor([T, 0, 1, 32, 33, 64])
    want = reference(*args, lengths=lengths)
    behind = torch.arange(T)[:, None] >= lengths[None]
    q, k, v, g, beta = (t.clone() for t in args[:5])
    for t in (q, k, v, g, beta):
        t[behind] = float("nan")
    heads = [(0, 1, 20, v), (0, 4, 40, g), (0, 11, 3, beta)]  # of three key heads, beside their neighbours
    for b, h, at, t in heads:
        t[at, b, h] = float("nan")
    y, state = run((q, k, v, g, beta, args[5]), lengths=lengths.cuda())
    for b, h, at, _ in heads:
        assert torch.isnan(y[at:, b, h]).all() and torch.isnan(state[b, h]).all()
        y[:, b, h], state[b, h] = 0, 0
        want[0][:, b, h], want[1][b, h] = 0, 0
    assert not y[behind.cuda()].any()
    check(y, state, want, T, 40 ** -0.5)


@pytest.mark.parametrize("T", [1, 96])
def test_captured_and_on_another_stream(T):
    args = make(T, 2, 1, 2, 128, 64, BF16, seed=12)
    want = reference(*args)
    q, k, v, g, beta, state = (t.cuda() for t in args)
    y, new, ws = torch.zeros_like(v), torch.zeros_like(state), binding.delta_rule_workspace(q, k, v)
    call = lambda: binding.delta_rule(q, k, v, g, beta, state=state, new_state=new, normalize=True, y=y, workspace=ws)  # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    check(y, new, want, T, 128 ** -0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        state.copy_(args[5].cuda() * (i + 1))
        y.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), new.clone()
        check(*got, reference(*args[:5], args[5] * (i + 1)), T, 128 ** -0.5)
        call()
        assert torch.equal(got[0], y) and torch.equal(got[1], new)


def test_refusals_of_the_binding():
    q, k, v, g, beta, state = (t.cuda() for t in make(4, 2, 1, 2, 64, 32, BF16))
    for bad in (lambda: binding.delta_rule(q, k, v, g.double(), beta), lambda: binding.delta_rule(q, k[:3], v, g, beta),
                lambda: binding.delta_rule(q.float(), k, v, g, beta), lambda: binding.delta_rule(q, k, v, g[:3], beta),
                lambda: binding.delta_rule(q, k, v, g, beta, state=state.half()), lambda: binding.delta_rule(q, k, v, g, beta, state=state[:1]),
                lambda: binding.delta_rule(q, k, v, g, beta, y=v.float()), lambda: binding.delta_rule(q, k, v, g.cpu(), beta),
                lambda: binding.delta_rule(q, k, v, g, beta, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(ValueError):
        binding.delta_rule(q, k, v.transpose(2, 3).contiguous().transpose(2, 3), g, beta)
    with pytest.raises(binding.LstmIntError):
        binding.delta_rule(q.expand(-1, -1, 3, -1), k.expand(-1, -1, 3, -1), v, g, beta)
