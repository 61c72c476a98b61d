"""include/lm_ops.h without a GPU: every declared symbol is there and bound, structs have the header's fields, refusals
come before any device work, and a host-only 4-bit model quantizes as the header says."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from paper_2101_05453_amd import binding

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lm_ops.h")).read()
CODE = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
BUF = (C.c_char * 4096)()
P = C.addressof(BUF)


def test_symbols_are_exported_and_bound():
    L, _ = binding.lm_lib()
    names = sorted(set(re.findall(r"\b((?:rms_norm|w4_linear|delta_rule)_[a-z_]+)\s*\(", CODE)))
    assert len(names) == 7
    for n in names:
        assert hasattr(L, n) and getattr(L, n).argtypes is not None, n


@pytest.mark.parametrize("struct, cls", [("rms_norm_args", binding.RmsNormArgs), ("w4_linear_params", binding.W4LinearParams),
                                         ("w4_linear_quant", binding.W4LinearQuant), ("delta_rule_args", binding.DeltaRuleArgs)])
def test_struct_fields_match_the_header(struct, cls):
    body = re.search(r"typedef struct \{([^}]*)\} " + struct + ";", CODE).group(1)
    fields = [re.sub(r"\[.*", "", name.strip().split()[-1].lstrip("*")) for decl in body.split(";") if decl.strip()
              for name in decl.split(",")]
    assert fields == [f[0] for f in cls._fields_]


def norm(device=0, x=P, residual=None, gate=None, weight=P, codes=P, scales=P, y=None, new_residual=None, null_args=False, **kw):
    a = dict(rows=2, cols=64, groups=1, dtype=binding.LM_BF16, zero_point=0, eps=1e-6, scale=0.0, x_stride=64, residual_stride=64,
             gate_stride=64, new_residual_stride=64)
    a.update(kw)
    args = None if null_args else binding.RmsNormArgs(**a)
    return binding.lm_lib()[0].rms_norm_forward(device, args, x, residual, gate, weight, codes, scales, y, new_residual, None)


@pytest.mark.parametrize("kw, code", [
    (dict(null_args=True), binding.E_INVALID_ARG), (dict(device=-1), binding.E_INVALID_ARG), (dict(x=None), binding.E_INVALID_ARG),
    (dict(weight=None), binding.E_INVALID_ARG), (dict(codes=None), binding.E_INVALID_ARG), (dict(scales=None), binding.E_INVALID_ARG),
    (dict(new_residual=P), binding.E_INVALID_ARG), (dict(rows=-1), binding.E_INVALID_ARG), (dict(cols=-64), binding.E_INVALID_ARG),
    (dict(groups=0), binding.E_INVALID_ARG), (dict(groups=3), binding.E_INVALID_ARG), (dict(dtype=3), binding.E_INVALID_ARG),
    (dict(dtype=-1), binding.E_INVALID_ARG), (dict(zero_point=128, scale=1.0), binding.E_INVALID_ARG),
    (dict(zero_point=-129, scale=1.0), binding.E_INVALID_ARG), (dict(x_stride=63), binding.E_INVALID_ARG),
    (dict(residual=P, residual_stride=63), binding.E_INVALID_ARG), (dict(gate=P, gate_stride=0), binding.E_INVALID_ARG),
    (dict(residual=P, new_residual=P, new_residual_stride=63), binding.E_INVALID_ARG),
    (dict(eps=0.0), binding.E_BAD_RANGE), (dict(eps=float("nan")), binding.E_BAD_RANGE), (dict(eps=float("inf")), binding.E_BAD_RANGE),
    (dict(scale=-1.0), binding.E_BAD_RANGE), (dict(scale=float("nan")), binding.E_BAD_RANGE),
    (dict(scale=float("inf")), binding.E_BAD_RANGE), (dict(cols=32769, rows=1), binding.E_UNSUPPORTED),
    (dict(rows=1 << 31), binding.E_UNSUPPORTED), (dict(cols=8208, groups=2, rows=1), binding.E_UNSUPPORTED),
    (dict(groups=16), binding.E_UNSUPPORTED), (dict(cols=8192, groups=2, rows=1), binding.E_UNSUPPORTED),
    (dict(rows=0), binding.OK), (dict(cols=0, x_stride=0), binding.OK), (dict(rows=0, x=None, weight=None), binding.OK)])
def test_norm_refusals(kw, code):
    assert norm(**kw) == code


def delta(device=0, q=P, k=P, v=P, g=P, beta=P, lengths=None, state=None, new_state=None, y=P, workspace=None, workspace_bytes=0,
          null_args=False, **kw):
    a = dict(steps=2, batch=1, key_heads=2, value_heads=4, key_dim=8, value_dim=8, dtype=binding.LM_F32, normalize=0, scale=1.0)
    a.update(kw)
    args = None if null_args else binding.DeltaRuleArgs(**a)
    return binding.lm_lib()[0].delta_rule_forward(device, args, q, k, v, g, beta, lengths, state, new_state, y, workspace,
                                                  workspace_bytes, None)


@pytest.mark.parametrize("kw, code", [
    (dict(null_args=True), binding.E_INVALID_ARG), (dict(device=-1), binding.E_INVALID_ARG), (dict(steps=-1), binding.E_INVALID_ARG),
    (dict(batch=-1), binding.E_INVALID_ARG), (dict(key_heads=0), binding.E_INVALID_ARG), (dict(value_heads=0), binding.E_INVALID_ARG),
    (dict(value_heads=3), binding.E_INVALID_ARG), (dict(value_heads=1), binding.E_INVALID_ARG), (dict(key_dim=0), binding.E_INVALID_ARG),
    (dict(value_dim=0), binding.E_INVALID_ARG), (dict(dtype=7), binding.E_INVALID_ARG), (dict(normalize=2), binding.E_INVALID_ARG),
    (dict(q=None), binding.E_INVALID_ARG), (dict(k=None), binding.E_INVALID_ARG), (dict(v=None), binding.E_INVALID_ARG),
    (dict(g=None), binding.E_INVALID_ARG), (dict(beta=None), binding.E_INVALID_ARG), (dict(y=None), binding.E_INVALID_ARG),
    (dict(scale=float("nan")), binding.E_BAD_RANGE), (dict(scale=float("inf")), binding.E_BAD_RANGE),
    (dict(key_dim=257), binding.E_UNSUPPORTED), (dict(value_dim=257), binding.E_UNSUPPORTED),
    (dict(batch=1 << 19), binding.E_UNSUPPORTED), (dict(steps=(1 << 24) + 1), binding.E_UNSUPPORTED),
    (dict(batch=0), binding.OK), (dict(steps=0), binding.OK)])
def test_delta_rule_refusals(kw, code):
    assert delta(**kw) == code


def test_delta_rule_workspace_is_asked_for():
    a = dict(steps=4096, batch=2, key_heads=2, value_heads=4, key_dim=128, value_dim=128, dtype=binding.LM_BF16, normalize=1, scale=1.0)
    need = binding.lm_lib()[0].delta_rule_workspace_bytes(binding.DeltaRuleArgs(**a))
    if need:
        at = (P + 255) & ~255
        assert delta(**a) == binding.E_WORKSPACE
        assert delta(workspace=at, workspace_bytes=need - 1, **a) == binding.E_WORKSPACE
        assert delta(workspace=at + 128, workspace_bytes=need, **a) == binding.E_WORKSPACE
    a["key_dim"] = 0
    assert binding.lm_lib()[0].delta_rule_workspace_bytes(binding.DeltaRuleArgs(**a)) == 0
    assert binding.lm_lib()[0].delta_rule_workspace_bytes(None) == 0


@pytest.mark.parametrize("K, group", [(64, 64), (75, 32), (300, 128), (1, 32), (128, 64)])
def test_w4_quantizes_floats(K, group):
    rng = np.random.default_rng(K)
    W = rng.standard_normal((13, K)).astype(np.float32)
    W[3] = 0
    q = binding.w4_prepare(W=W, group=group, device=-1).get_quant()
    groups = -(-K // group)
    assert q["group_size"] == group and q["codes"].shape == (13, K) and q["scales"].shape == (13, groups)
    padded = np.zeros((13, groups * group), np.float32)
    padded[:, :K] = W
    s = np.abs(padded.reshape(13, groups, group)).max(2) / np.float32(7)
    assert (q["scales"] == s).all()
    each = np.repeat(s, group, 1)[:, :K]
    ratio = np.divide(W, each, out=np.zeros_like(W), where=each > 0)
    assert (q["codes"] == np.copysign(np.floor(np.abs(ratio) + np.float32(0.5)), ratio)).all()
    assert np.abs(q["codes"]).max() == 7


def test_w4_keeps_given_codes():
    rng = np.random.default_rng(1)
    codes, scales = rng.integers(-8, 8, (5, 70)).astype(np.int8), rng.standard_normal((5, 3)).astype(np.float32)
    q = binding.w4_prepare(codes=codes, scales=scales, group=32, device=-1).get_quant()
    assert (q["codes"] == codes).all() and (q["scales"] == scales).all()


def w4_prepare(**kw):
    one = np.ones(1 << 12, np.float32)
    ones8 = np.ones(1 << 12, np.int8)
    fp = one.ctypes.data_as(C.POINTER(C.c_float))
    cp = ones8.ctypes.data_as(C.POINTER(C.c_int8))
    a = dict(inputs=64, outputs=4, group_size=32, W=fp, codes=None, scales=None, bias=None)
    edit = kw.pop("edit", None)
    a.update({k: fp if v == "f" else cp if v == "c" else v for k, v in kw.items()})
    if edit:
        edit(one, ones8)
    h = C.c_void_p()
    rc = binding.lm_lib()[0].w4_linear_prepare(binding.W4LinearParams(**a), -1, C.byref(h))
    assert bool(h.value) == (rc == binding.OK)
    binding.lm_lib()[0].w4_linear_destroy(h)
    return rc


@pytest.mark.parametrize("kw, code", [
    (dict(), binding.OK), (dict(W=None, codes="c", scales="f", bias="f"), binding.OK),
    (dict(inputs=0), binding.E_INVALID_ARG), (dict(outputs=0), binding.E_INVALID_ARG), (dict(group_size=16), binding.E_INVALID_ARG),
    (dict(group_size=0), binding.E_INVALID_ARG), (dict(W=None), binding.E_INVALID_ARG), (dict(codes="c"), binding.E_INVALID_ARG),
    (dict(scales="f"), binding.E_INVALID_ARG), (dict(W=None, codes="c"), binding.E_INVALID_ARG),
    (dict(W=None, codes="c", scales="f", edit=lambda f, c: c.__setitem__(9, 8)), binding.E_INVALID_ARG),
    (dict(W=None, codes="c", scales="f", edit=lambda f, c: c.__setitem__(9, -9)), binding.E_INVALID_ARG),
    (dict(W=None, codes="c", scales="f", edit=lambda f, c: f.__setitem__(1, np.nan)), binding.E_BAD_RANGE),
    (dict(edit=lambda f, c: f.__setitem__(70, np.inf)), binding.E_BAD_RANGE),
    (dict(edit=lambda f, c: f.__setitem__(0, np.nan)), binding.E_BAD_RANGE),
    (dict(inputs=(1 << 17) + 1), binding.E_UNSUPPORTED), (dict(outputs=(1 << 24) + 1), binding.E_UNSUPPORTED)])
def test_w4_prepare_refusals(kw, code):
    assert w4_prepare(**kw) == code


def test_w4_forward_refusals():
    L, _ = binding.lm_lib()
    m = binding.w4_prepare(W=np.ones((4, 64), np.float32), group=32, device=-1)

    def forward(h=m._h, x=P, x_stride=64, rows=2, scales=None, zp=0, y=P, y_stride=4, dtype=binding.LM_F32):
        return L.w4_linear_forward(h, x, x_stride, rows, scales, 1.0, zp, y, y_stride, dtype, None)

    assert forward() == binding.E_DEVICE and forward(rows=0) == binding.OK
    for kw in (dict(h=None), dict(x=None), dict(y=None), dict(rows=-1), dict(x_stride=63), dict(y_stride=3), dict(zp=128), dict(zp=-129),
               dict(dtype=3)):
        assert forward(**kw) == binding.E_INVALID_ARG, kw
    assert L.w4_linear_prepare(None, -1, None) == binding.E_INVALID_ARG
    assert L.w4_linear_get_quant(None, None) == binding.E_INVALID_ARG
    L.w4_linear_destroy(None)


def test_binding_refuses_what_the_library_cannot_see():
    import torch

    x = torch.zeros(2, 64)
    with pytest.raises(AssertionError):
        binding.rms_norm(x, torch.ones(64))  # not on a GPU
    with pytest.raises(AssertionError):
        binding.delta_rule(*[torch.zeros(1, 1, 1, 8)] * 3, torch.zeros(1, 1, 1), torch.zeros(1, 1, 1))
