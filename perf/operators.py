"""Timed cases of the operators around the recurrent cells: root-mean-square norm into int8 codes, products with 4-bit
weights, the gated delta rule.

A case names an operator ("op") and its sizes.  `prepare` makes from the seed what a program holds before the call:
activations, weights in 4 bits with their scales, the cell's state.  `run` makes one pass, in elementary torch operations,
or through the package's entry points where `own` is set."""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
CHUNK = 64  # steps that the plain form of the delta rule takes at a time


def _norm(name, rows, cols, dtype, heads=1, residual=False, gate=False, static=False):
    """heads: the norm is taken over cols / heads columns each.  static: codes at a fixed scale and zero point, as a
    recurrent layer reads them; otherwise a scale of each row."""
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "heads": heads, "residual": residual,
            "gate": gate, "static": static}


def _w4(name, rows, inputs, outputs, group, dtype, static=False, bias=False):
    """static: activations with one scale and a zero point, as a recurrent layer returns them; otherwise a scale of each row."""
    return {"name": name, "op": "w4", "rows": rows, "inputs": inputs, "outputs": outputs, "group": group, "dtype": dtype,
            "static": static, "bias": bias}


def _delta(name, steps, batch, key_heads, value_heads, key_dim, value_dim, dtype, normalize=True, ragged=False):
    """ragged: the batch's sequences have lengths of their own, an empty one among them."""
    return {"name": name, "op": "delta", "steps": steps, "batch": batch, "key_heads": key_heads, "value_heads": value_heads,
            "key_dim": key_dim, "value_dim": value_dim, "dtype": dtype, "normalize": normalize, "ragged": ragged}


def listed():
    return [
        # the norm before a product for a single token: latency
        _norm("norm_1x2048", 1, 2048, "bf16", residual=True),
        # features of many odd rows into the codes that a recurrent layer reads
        _norm("norm_9999x1001_static", 9999, 1001, "fp16", residual=True, static=True),
        # the gated norm of each head behind the delta rule, a long prompt
        _norm("norm_8192x32x128_gated", 8192, 4096, "bf16", heads=32, gate=True),
        # a projection for a single token
        _w4("w4_1x2048x2048", 1, 2048, 2048, 128, "bf16"),
        # an output layer over a vocabulary of odd size, on the codes that a projected recurrent layer returns
        _w4("w4_7x640x32003_static", 7, 640, 32003, 32, "fp32", static=True, bias=True),
        # a decoding step of a batch
        _w4("w4_32x4096x4096", 32, 4096, 4096, 64, "fp16"),
        # a whole batch of sequences: the gates' width of an encoder layer
        _w4("w4_16384x640x8192", 16384, 640, 8192, 128, "bf16"),
        # one step for one sequence
        _delta("delta_step_b1", 1, 1, 4, 8, 128, 128, "bf16"),
        # one step for a serving batch
        _delta("delta_step_b64", 1, 64, 8, 16, 128, 128, "bf16"),
        # one long prompt: few heads, a long way through time
        _delta("delta_4096_b1", 4096, 1, 8, 16, 128, 128, "bf16"),
        # sequences of unlike lengths, sizes that no tile divides, in full precision
        _delta("delta_777_b5_ragged", 777, 5, 3, 6, 96, 80, "fp32", ragged=True),
        # a batch of prompts
        _delta("delta_2048_b8", 2048, 8, 16, 32, 128, 128, "bf16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    def width(lo, hi):  # multiples of 64 or 8 as models have them, and any size
        n, kind = spread(lo, hi), rng.random()
        if kind < 0.5:
            n = round(n / 64) * 64 if n >= 64 else round(n / 16) * 16
        elif kind < 0.75:
            n = round(n / 8) * 8
        return max(lo, min(hi, n))

    op, dtype = rng.choice(["norm", "w4", "w4", "delta", "delta", "delta"]), rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while True:
        if op == "norm":
            heads = rng.choice([1, 1, rng.randint(2, 32)])
            cols = heads * width(16, max(16, 8192 // heads)) if heads > 1 else width(16, 8192)
            c = _norm(None, spread(1, 32768), cols, dtype, heads=heads, residual=heads == 1 and rng.random() < 0.6,
                      gate=heads > 1 and rng.random() < 0.7, static=rng.random() < 0.3)
            fits = c["rows"] * cols <= 2 ** 25
        elif op == "w4":
            static = rng.random() < 0.3
            c = _w4(None, spread(1, 16384) if rng.random() < 0.4 else spread(1, 64), width(32, 8192), width(16, 32768),
                    rng.choice([32, 64, 128]), dtype, static=static, bias=static or rng.random() < 0.2)
            fits = (c["rows"] * c["inputs"] * c["outputs"] <= 16384 * 640 * 8192 and c["inputs"] * c["outputs"] <= 2 ** 25 and
                    c["rows"] * c["outputs"] <= 2 ** 26)
        else:
            heads, shared = spread(1, 16), rng.choice([1, 1, 2, 4])
            c = _delta(None, 1 if rng.random() < 0.25 else spread(1, 4096), spread(1, 64), heads, heads * shared,
                       rng.choice([64, 128, 128, width(16, 256)]), rng.choice([64, 128, 128, width(16, 256)]), dtype,
                       normalize=rng.random() < 0.8, ragged=rng.random() < 0.3)
            state = c["batch"] * c["value_heads"] * c["key_dim"] * c["value_dim"]
            fits = c["steps"] * state <= 2 ** 31 and state <= 2 ** 24
        if fits:
            del c["name"]
            return c


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        streams = 1 + 2 * case["residual"] + case["gate"]  # read, the sum written; the gate
        return {"bytes": n * (streams * size + 1) + 4 * case["cols"] // case["heads"] + (0 if case["static"] else 4 * case["rows"]),
                "flops": n * (5 + 5 * case["gate"])}
    if case["op"] == "w4":
        M, K, N = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": N * K // 2 + 4 * N * -(-K // case["group"]) + M * K + M * N * size + 4 * N * case["bias"] +
                (0 if case["static"] else 4 * M), "flops": 2 * M * N * K}
    tokens = case["steps"] * case["batch"] * (0.6 if case["ragged"] else 1)  # mean length of a ragged batch
    cells = case["batch"] * case["value_heads"] * case["key_dim"] * case["value_dim"]
    row = 2 * case["key_heads"] * case["key_dim"] * size + 2 * case["value_heads"] * case["value_dim"] * size + 8 * case["value_heads"]
    # per step and cell of the state: decay, S'k, the update, S'q
    return {"bytes": tokens * row + 8 * cells, "flops": 7 * tokens * cells / case["batch"]}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def prepare(case, seed):
    g, dt = _generator(seed), TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(shape, generator=g, device="cuda")

    s = SimpleNamespace(case=case)
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # a few columns and rows are louder than others, as hidden states are
        loud = torch.exp(0.5 * normal(cols)) * uniform(0.5, 2.0, rows, 1)
        s.x = (normal(rows, cols) * loud).to(dt)
        s.residual = (2 * normal(rows, cols) * loud).to(dt) if case["residual"] else None
        s.gate = normal(rows, cols).to(dt) if case["gate"] else None
        s.weight = uniform(0.5, 1.5, cols // case["heads"])
        s.scale, s.zero_point = (0.04, -3) if case["static"] else (None, 0)
    elif case["op"] == "w4":
        M, K, N, G = case["rows"], case["inputs"], case["outputs"], case["group"]
        w = normal(N, -(-K // G) * G) / math.sqrt(K)
        w[:, K:] = 0
        w = w.view(N, -1, G)
        s.scales = w.abs().amax(2) / 7
        s.codes = torch.round(w / s.scales.clamp_min(1e-30)[:, :, None]).clamp_(-8, 7).view(N, -1)[:, :K].to(torch.int8).contiguous()
        s.x = (normal(M, K) * 36).round().clamp_(-128 if case["static"] else -127, 127).to(torch.int8)
        s.x_scale, s.zero_point = (0.0123, 5) if case["static"] else (uniform(0.005, 0.05, M), 0)
        s.bias = uniform(-1, 1, N) if case["bias"] else None
        if own:  # the handle with the weights laid out, which a program makes once; the inputs do not go by it
            from paper_2101_05453_amd import binding
            s.handle = binding.w4_prepare(codes=s.codes.cpu().numpy(), scales=s.scales.cpu().numpy(), group=G,
                                          bias=None if s.bias is None else s.bias.cpu().numpy())
    else:
        T, B, Hk, Hv, Dk, Dv = (case[k] for k in ("steps", "batch", "key_heads", "value_heads", "key_dim", "value_dim"))
        # q, k and v as one projection writes them: side by side in its rows
        qkv = normal(T, B, 2 * Hk * Dk + Hv * Dv)
        if not case["normalize"]:
            qkv[:, :, :2 * Hk * Dk] /= math.sqrt(Dk)
        qkv = qkv.to(dt)
        s.q, s.k = (qkv[:, :, i * Hk * Dk:(i + 1) * Hk * Dk].view(T, B, Hk, Dk) for i in (0, 1))
        s.v = qkv[:, :, 2 * Hk * Dk:].view(T, B, Hv, Dv)
        s.g = -torch.exp(uniform(-7, 0.5, 1, 1, Hv)) * uniform(0.2, 2.0, T, B, Hv)  # slow heads and quick ones
        s.beta = torch.sigmoid(normal(T, B, Hv))
        s.state = normal(B, Hv, Dk, Dv) / math.sqrt(Dk)
        s.new_state = torch.empty_like(s.state)
        s.lengths = None
        if case["ragged"]:
            s.lengths = (uniform(0.2, 1.0, B) * T).ceil().to(torch.int32)
            s.lengths[-1] = 0 if B > 1 else T
        # outputs behind the end of a sequence stay as they were: zeros here
        s.y = torch.zeros(T, B, Hv, Dv, dtype=dt, device="cuda") if case["ragged"] else torch.empty(T, B, Hv, Dv, dtype=dt, device="cuda")
        if own:  # scratch memory that a program keeps
            from paper_2101_05453_amd import binding
            s.workspace = binding.delta_rule_workspace(s.q, s.k, s.v)
    return s


def run(s):
    return _own(s) if own else {"norm": _plain_norm, "w4": _plain_w4, "delta": _plain_delta}[s.case["op"]](s)


def _own(s):
    from paper_2101_05453_amd import binding

    if s.case["op"] == "norm":
        heads, new_residual = s.case["heads"], torch.empty_like(s.x) if s.case["residual"] else None
        codes, scales = binding.rms_norm_quantize(s.x, s.weight, eps=EPS, groups=heads, residual=s.residual, new_residual=new_residual,
                                                  gate=s.gate, scale=s.scale, zero_point=s.zero_point)
        values = (codes - float(s.zero_point)) * s.scale if s.case["static"] else codes * scales[:, None]
        return {"values": values, "residual": new_residual}
    if s.case["op"] == "w4":
        return s.handle.forward(s.x, s.x_scale, zero_point=s.zero_point, dtype=TYPES[s.case["dtype"]])
    binding.delta_rule(s.q, s.k, s.v, s.g, s.beta, state=s.state, new_state=s.new_state, lengths=s.lengths,
                       normalize=s.case["normalize"], y=s.y, workspace=s.workspace)
    return {"y": s.y, "state": s.new_state}


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_norm(s):
    # a code is decided next to the border between two: 64 bits
    rows, cols = s.x.shape
    r = s.x.double() + s.residual.double() if s.case["residual"] else s.x.double()
    n = r.view(rows, s.case["heads"], -1)
    n = (n * torch.rsqrt((n * n).mean(2, keepdim=True) + EPS) * s.weight.double()).view(rows, cols)
    if s.case["gate"]:
        z = s.gate.double()
        n = n * (z / (1 + torch.exp(-z)))
    if s.case["static"]:
        codes = (torch.floor(n / s.scale + 0.5) + s.zero_point).clamp(-128, 127)
        values = (codes.float() - s.zero_point) * s.scale
    else:
        most = n.abs().amax(1, keepdim=True)
        codes = torch.floor(n * (127 / most) + 0.5)
        values = codes.float() * (most / 127).float()
    return {"values": values, "residual": r.to(s.x.dtype) if s.case["residual"] else None}


def _plain_w4(s):
    N, K = s.codes.shape
    w = s.codes.float() * s.scales.repeat_interleave(s.case["group"], 1)[:, :K]
    if s.case["static"]:
        y = ((s.x.float() - s.zero_point) * s.x_scale) @ w.T
    else:
        y = (s.x.float() @ w.T) * s.x_scale[:, None]
    return (y if s.bias is None else y + s.bias).to(TYPES[s.case["dtype"]])


def _unit_lower_inverse(below):
    # (1 + below)^-1 by blocks on the diagonal of twice the size each time: (D + L)^-1 = D^-1 - D^-1 L D^-1, as L D^-1 L = 0
    C = below.shape[-1]
    at, inverse, size = torch.arange(C, device=below.device), torch.eye(C, device=below.device), 1
    while size < C:
        same, other = at // (2 * size), at // size
        inverse = inverse - inverse @ (below * ((same[:, None] == same) & (other[:, None] != other))) @ inverse
        size *= 2
    return inverse


def _plain_delta(s):
    # CHUNK steps at a time: inside a chunk the updates u are the solution of a triangular system, between chunks the
    # state is carried
    T, B, Hv, Dv = s.v.shape
    Dk, shared, C = s.k.shape[3], Hv // s.k.shape[2], min(CHUNK, T)
    chunks = -(-T // C)

    def split(x):  # [T, B, H, ...] -> [B, H, chunks, C, ...], zeros behind the end
        x = torch.cat([x, x.new_zeros((chunks * C - T, *x.shape[1:]))]) if chunks * C > T else x
        return x.reshape(chunks, C, *x.shape[1:]).permute(2, 3, 0, 1, *range(4, x.dim() + 1))

    q, k, v, g, beta = s.q.float(), s.k.float(), s.v.float(), s.g.double(), s.beta
    if s.lengths is not None:
        inside = torch.arange(T, device=v.device)[:, None] < s.lengths[None]
        g, beta, k = g * inside[:, :, None], beta * inside[:, :, None], k * inside[:, :, None, None]
    if s.case["normalize"]:
        q = q * torch.rsqrt((q * q).sum(3, keepdim=True) + EPS)
        k = k * torch.rsqrt((k * k).sum(3, keepdim=True) + EPS)
    if T == 1:  # a single step: the recurrence as it stands
        q, k = (x[0].repeat_interleave(shared, 1)[..., None] for x in (q / math.sqrt(Dk), k))
        state = s.state * torch.exp(g[0].float())[..., None, None]
        u = beta[0][..., None] * (v[0] - (state * k).sum(2))
        state = state + k * u[:, :, None]
        y = (state * q).sum(2)[None]
        return {"y": (y if s.lengths is None else y * inside[:, :, None, None]).to(s.v.dtype), "state": state}
    q, k = ((split(x).repeat_interleave(shared, 1)) for x in (q / math.sqrt(Dk), k))
    v, g, beta = split(v), split(g), split(beta)[..., None]
    c = g.cumsum(3)  # log of the decay since the chunk began: a long sum, 64 bits
    between = torch.exp((c[..., :, None] - c[..., None, :]).float()).tril()
    since, left = torch.exp(c.float())[..., None], torch.exp((c[..., -1:] - c).float())[..., None]
    kt = k.transpose(3, 4).contiguous()
    inverse = _unit_lower_inverse((beta * between * (k @ kt)).tril(-1))
    u0, w = inverse @ (beta * v), inverse @ (beta * since * k)
    inside_chunk, q, kt = between * (q @ kt), q * since, kt * left.transpose(3, 4)
    whole, state, ys = since[..., -1:, :], s.state, []
    for i in range(chunks):
        u = u0[:, :, i] - w[:, :, i] @ state
        ys.append(q[:, :, i] @ state + inside_chunk[:, :, i] @ u)
        state = whole[:, :, i] * state + kt[:, :, i] @ u
    y = torch.stack(ys, 2).reshape(B, Hv, chunks * C, Dv)[:, :, :T].permute(2, 0, 1, 3)
    if s.lengths is not None:
        y = y * inside[:, :, None, None]
    return {"y": y.to(s.v.dtype).contiguous(), "state": state}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare({k: v for k, v in case.items()}, seed)
    if case["op"] == "norm":
        r = s.x.double() if s.residual is None else s.x.double() + s.residual.double()
        per_head = r.reshape(case["rows"] * case["heads"], -1)
        n = per_head / torch.sqrt(per_head.pow(2).sum(1, keepdim=True) / per_head.shape[1] + EPS) * s.weight.double()
        n = n.reshape(r.shape)
        if s.gate is not None:
            n = n * s.gate.double() * torch.sigmoid(s.gate.double())
        if case["static"]:
            codes = torch.clamp(torch.floor(n / s.scale + 0.5) + s.zero_point, -128, 127)
            values = (codes - s.zero_point) * s.scale
        else:
            step = n.abs().max(1, keepdim=True).values / 127
            values = torch.floor(n / step + 0.5) * step
        return {"values": values, "residual": r if case["residual"] else None}
    if case["op"] == "w4":
        group_of = torch.arange(case["inputs"], device="cuda") // case["group"]
        x = s.x.double() - s.zero_point
        x = x * (s.x_scale if case["static"] else s.x_scale.double()[:, None])
        y = torch.mm(x, (s.codes.double() * s.scales.double()[:, group_of]).t())
        return y if s.bias is None else y + s.bias.double()
    # the recurrence step by step
    T, B, Hv, Dv = s.v.shape
    head = torch.arange(Hv, device="cuda") // (Hv // case["key_heads"])
    S, y = s.state.double(), torch.zeros(T, B, Hv, Dv, dtype=torch.float64, device="cuda")
    for t in range(T):
        q, k = s.q[t].double(), s.k[t].double()
        if case["normalize"]:
            q, k = (x / torch.sqrt(x.pow(2).sum(2, keepdim=True) + EPS) for x in (q, k))
        q, k = q[:, head, :, None] * case["key_dim"] ** -0.5, k[:, head, :, None]
        decayed = S * torch.exp(s.g[t].double())[:, :, None, None]
        u = s.beta[t].double()[:, :, None] * (s.v[t].double() - (decayed * k).sum(2))
        new = decayed + k * u[:, :, None, :]
        out = (new * q).sum(2)
        if s.lengths is None:
            S, y[t] = new, out
        else:
            live = (s.lengths > t)[:, None, None]
            S, y[t] = torch.where(live[..., None], new, S), out * live
    return {"y": y, "state": S}
