"""include/lm_ops.h without a GPU: outputs that would be written over each other are refused before any device work."""
import ctypes as C

import pytest

from paper_2101_05453_amd import binding

BUF = (C.c_char * 4096)()
P = C.addressof(BUF)


def delta(y_stride, device=0, **kw):
    a = dict(steps=2, batch=3, key_heads=2, value_heads=4, key_dim=8, value_dim=8, dtype=binding.LM_F32, normalize=0, scale=1.0)
    a.update(kw)
    args = binding.DeltaRuleArgs(**a, y_stride=(C.c_int64 * 3)(*y_stride))
    return binding.lm_lib()[0].delta_rule_forward(device, args, P, P, P, P, P, None, None, None, P, None, 0, None)


# no device has the number 4096: what is not refused as an argument ends there
@pytest.mark.parametrize("kw, code", [
    (dict(y_stride=(96, 32, 8)), binding.E_DEVICE), (dict(y_stride=(32, 64, 8)), binding.E_DEVICE), (dict(y_stride=(-96, -32, -8)), binding.E_DEVICE),
    (dict(y_stride=(0, 32, 8), steps=1), binding.E_DEVICE), (dict(y_stride=(96, 3, 8), batch=1), binding.E_DEVICE),
    (dict(y_stride=(96, 8, 1), value_heads=1, key_heads=1), binding.E_DEVICE),
    (dict(y_stride=(0, 32, 8)), binding.E_INVALID_ARG), (dict(y_stride=(96, 0, 8)), binding.E_INVALID_ARG),
    (dict(y_stride=(96, 32, 0)), binding.E_INVALID_ARG), (dict(y_stride=(96, 32, 7)), binding.E_INVALID_ARG),
    (dict(y_stride=(7, 32, 8)), binding.E_INVALID_ARG), (dict(y_stride=(96, 32, -7)), binding.E_INVALID_ARG)])
def test_delta_rule_outputs_over_each_other(kw, code):
    assert delta(device=4096, **kw) == code
