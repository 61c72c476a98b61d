"""The operators of lm_ops.h as a model runs them: a block around the delta rule (norm, 4-bit projection, delta rule, gated
norm of each head, 4-bit projection), whole sequences and step by step, and in front of and behind an integer LSTM."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import float_reference  # noqa: E402
import lstm_workloads as wl  # noqa: E402
from paper_2101_05453_amd import binding  # noqa: E402

W, HK, HV, D = 192, 2, 4, 64  # width of the residual, key and value heads, their dimension
BF16 = torch.bfloat16


def weights(n, k, seed):
    return (np.random.default_rng(seed).standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)


class Block:
    def __init__(self):
        g = torch.Generator().manual_seed(1)
        self.norm, self.head_norm = (torch.rand(n, generator=g).add(0.5).cuda() for n in (W, D))
        self.qkv = binding.w4_prepare(W=weights(2 * HK * D + HV * D, W, 2), group=64)
        self.z = binding.w4_prepare(W=weights(HV * D, W, 3), group=64)
        self.rates = binding.w4_prepare(W=weights(2 * HV, W, 4), group=32)
        self.out = binding.w4_prepare(W=weights(W, HV * D, 5), group=128)

    def __call__(self, x, residual, state):
        """x, residual [T, B, W]; returns what the block adds, the residual, and the outputs of every stage"""
        new = torch.empty_like(residual)
        codes, scales = binding.rms_norm_quantize(x, self.norm, residual=residual, new_residual=new)
        qkv = self.qkv.forward(codes, scales)
        q, k = (qkv[..., i * HK * D:(i + 1) * HK * D].unflatten(2, (HK, D)) for i in (0, 1))
        v = qkv[..., 2 * HK * D:].unflatten(2, (HV, D))
        z = self.z.forward(codes, scales)
        rates = self.rates.forward(codes, scales, dtype=torch.float32)
        g, beta = -torch.nn.functional.softplus(rates[..., :HV]), torch.sigmoid(rates[..., HV:])
        y = binding.delta_rule(q, k, v, g, beta, state=state, normalize=True).flatten(2)
        codes2, scales2 = binding.rms_norm_quantize(y, self.head_norm, gate=z, groups=HV)
        return self.out.forward(codes2, scales2), new, dict(codes=codes, scales=scales, qkv=qkv, z=z, rates=rates, y=y, codes2=codes2, scales2=scales2)


def inputs(T, B, seed=7):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, B, W, generator=g).to(BF16).cuda() for _ in range(2))


def dequantized(m):
    q = m.get_quant()
    return torch.from_numpy(q["codes"].astype(np.float64) * np.repeat(q["scales"], q["group_size"], 1)[:, :m.inputs])


def test_block_against_its_definition_stage_by_stage():
    block, (x, res) = Block(), inputs(50, 3)
    state = torch.zeros(3, HV, D, D, device="cuda")
    add, new, s = block(x, res, state)
    c = {k: v.cpu() for k, v in s.items()}
    # codes are the definition's, one by one
    r = x.cpu().double() + res.cpu().double()
    n = r * torch.rsqrt(r.pow(2).mean(2, keepdim=True) + 1e-6) * block.norm.cpu().double()
    assert (c["codes"].double() == torch.floor(n / n.abs().amax(2, keepdim=True) * 127 + 0.5)).all()
    xq = c["codes"].double() * c["scales"].double()[..., None]
    # a product: bfloat16's one rounding, and float32 sums of a handful of groups
    for name, m in (("qkv", block.qkv), ("z", block.z)):
        want = xq @ dequantized(m).T
        assert ((c[name].double() - want).abs() <= want.abs() * 2.0 ** -8 + 1e-5).all()
    y, z = c["y"].double(), c["z"].double()
    n = y.unflatten(2, (HV, D))
    n = (n * torch.rsqrt(n.pow(2).mean(3, keepdim=True) + 1e-6) * block.head_norm.cpu().double()).flatten(2) * z / (1 + torch.exp(-z))
    assert (c["codes2"].double() == torch.floor(n / n.abs().amax(2, keepdim=True) * 127 + 0.5)).all()
    want = (c["codes2"].double() * c["scales2"].double()[..., None]) @ dequantized(block.out).T
    assert ((add.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + 1e-5).all()
    assert torch.equal(new.cpu(), r.to(BF16))


def test_a_prompt_and_then_single_steps_in_a_graph():
    T, B = 45, 4
    block, (x, res) = Block(), inputs(T + 6, B)
    whole_state = torch.zeros(B, HV, D, D, device="cuda")
    whole, _, ws = block(x, res, whole_state)
    state = torch.zeros_like(whole_state)
    _, _, first = block(x[:T].contiguous(), res[:T].contiguous(), state)
    xs, rs = torch.empty(1, B, W, dtype=BF16, device="cuda"), torch.empty(1, B, W, dtype=BF16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):  # once outside of the capture
        xs.copy_(x[T:T + 1])
        rs.copy_(res[T:T + 1])
        block(xs, rs, state.clone())
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        add, new, s = block(xs, rs, state)
    ys = [first["y"]]
    for t in range(T, T + 6):
        xs.copy_(x[t:t + 1])
        rs.copy_(res[t:t + 1])
        graph.replay()
        ys.append(s["y"].clone())
        assert torch.equal(s["codes"], ws["codes"][t:t + 1])  # rows do not depend on how many there are
    # The state took the same steps in chunks of 32 or one by one: float32 roundings, (8 + sqrt(64)) 2^-24 of the norms at
    # each of 51 steps, which differ on both sides; outputs one rounding to bfloat16 on each side besides.
    most = max(1.0, float(ws["qkv"].float().abs().max()) * D ** 0.5, float(whole_state.norm(dim=(2, 3)).max()))
    walk = 2 * 4 * (T + 7) ** 0.5 * 16 * 2.0 ** -24 * most
    assert float((state - whole_state).norm(dim=(2, 3)).max()) <= walk
    y, want = torch.cat(ys).float(), ws["y"].float()
    assert ((y - want).abs() <= want.abs() * 2.0 ** -7 + walk * D ** -0.5).all()
    assert whole.shape == (T + 6, B, W)


def test_around_an_integer_lstm(orc):
    """features -> norm at the model's input quantization -> integer LSTM -> 4-bit output layer on its codes"""
    layers, x = wl.make_custom([W], 128, 96, wl.LAYER_NORM | wl.PROJECTION, 5, 9, seed=3)
    norm = torch.ones(W)
    f = torch.from_numpy(x)
    n = f.double() * torch.rsqrt(f.double().pow(2).mean(2, keepdim=True) + 1e-6)
    float_reference.collect_statistics(layers, n.float().numpy())
    model, oracle_model = binding.prepare(layers), orc.prepare(layers)
    q = model.get_quant(0)
    codes, none = binding.rms_norm_quantize(f.cuda(), norm.cuda(), scale=q["s_x"], zero_point=q["zp_x"])
    assert none is None
    assert (codes.cpu().double() == (torch.floor(n / q["s_x"] + 0.5) + q["zp_x"]).clamp(-128, 127)).all()
    h = model.forward(codes)
    torch.cuda.synchronize()
    assert model.device_status() == 0
    assert (h.cpu().numpy() == orc.forward(oracle_model, codes.cpu().numpy())).all()
    bias = np.linspace(-1, 1, 1003).astype(np.float32)
    head = binding.w4_prepare(W=weights(1003, 96, 9), bias=bias, group=32)
    logits = head.forward(h, q["s_h"], zero_point=q["zp_h"], dtype=torch.float32)
    real = (h.cpu().double() - q["zp_h"]) * float(np.float32(q["s_h"]))
    want = real @ dequantized(head).T + torch.from_numpy(bias).double()
    terms = real.abs() @ dequantized(head).abs().T + 1
    assert logits.shape == (9, 5, 1003) and ((logits.cpu().double() - want).abs() <= terms * 6 * 2.0 ** -24).all()
