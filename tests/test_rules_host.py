"""Host-side checks of the decoding rules: what ee_logit_rules refuses is refused before any device work, and the
definition that the GPU tests compare with is pinned on small cases."""
import ctypes as C

import numpy as np
import pytest

import paper_2510_01336_amd as hs
from rules_common import adjust, pack, pick, softmax


def call(**over):
    """A call that would be accepted (addresses are never touched: the checks come first)."""
    c = hs.ee_rules_call()
    base = dict(n_seq=2, rows=3, vocab=100, dtype=hs.EE_F32, logits=4096, logits_stride=100, out=8192, out_stride=100, row_start=12288,
                workspace=16384, workspace_bytes=hs.ee_logit_rules_bytes(3, 100))
    base.update(over)
    for k, v in base.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("over, word", [
    (dict(rows=-1), "shape"), (dict(n_seq=-1), "shape"), (dict(vocab=0), "shape"), (dict(dtype=7), "dtype"),
    (dict(logits=None), "null"), (dict(out=None), "null"), (dict(row_start=None), "null"),
    (dict(logits=4098), "aligned"), (dict(out=8194), "aligned"), (dict(dtype=hs.EE_BF16, logits=4097), "aligned"),
    (dict(logits_stride=99), "strides"), (dict(out_stride=64), "strides"),
    (dict(out=4096, dtype=hs.EE_BF16), "in place"), (dict(out=4096, out_stride=104), "in place"),
    (dict(repetition=4096), "penalties"), (dict(tokens=4096, tokens_room=8, tokens_stride=8), "penalties"),
    (dict(tokens=4096, first_len=4096), "penalties"), (dict(tokens=4096, first_len=4096, tokens_room=8, tokens_stride=7), "penalties"),
    (dict(bias_start=4096, n_bias=1), "biases"), (dict(bias_token=4096), "biases"), (dict(bias_start=4096, n_bias=-1), "biases"),
    (dict(allowed=4096, allowed_stride=3, allowed_rows=3), "masks"), (dict(allowed=4096, allowed_stride=4, allowed_rows=2), "masks"),
    (dict(allowed_row=4096), "allowed_row"), (dict(workspace=None), "workspace"), (dict(workspace=16400), "workspace"),
    (dict(workspace_bytes=16), "workspace")], ids=lambda v: str(v)[:40])
def test_refusals(over, word):
    with pytest.raises(hs.EEError) as e:
        hs.ee_logit_rules(call(**over), 0)
    assert e.value.code == -1 and word in str(e.value), str(e.value)


def test_calls_without_rows_do_nothing():
    hs.ee_logit_rules(call(rows=0, logits=None, out=None, workspace=None), 0)
    hs.ee_logit_rules(call(n_seq=0, logits=None), 0)
    assert hs.lib.ee_logit_rules(None, None) == -1
    assert hs.ee_logit_rules_bytes(-1, 5) == 0 and hs.ee_logit_rules_bytes(4, 0) == 0 and hs.ee_logit_rules_bytes(0, 5) > 0


def test_session_rules_refuse_what_is_no_session():
    assert hs.lib.ee_rules_bytes(None, 0) == 0
    assert hs.lib.ee_rules_attach(None, 0, None, 0) == -1
    assert hs.lib.ee_rules_set(None, 0, None) == -1
    assert hs.lib.ee_rules_rows(None, 0, 0, None) == -1


def test_struct_layout():
    """Two independent sums of the header's fields on an LP64 host."""
    assert C.sizeof(hs.ee_rules_call) == 4 * 4 + 8 * 4 + 4 * 2 + 8 * 2 + 8 * 2 + 8 * 2 + 8 * 4 + 8 * 3 + 8 * 3 + 4 * 2 + 8 * 2
    assert C.sizeof(hs.ee_rules) == 16 + 8 + 24


def test_definition_on_small_cases():
    x = [2.0, -2.0, 1.0, 0.0]
    # seen tokens 0 and 1 (prompt), token 2 twice behind it
    assert adjust(x, [0, 1, 2, 2], 2, rho=2.0).tolist() == [1.0, -4.0, 0.5, 0.0]
    assert adjust(x, [0, 1, 2, 2], 2, freq=0.25, pres=1.0).tolist() == [2.0, -2.0, -0.5, 0.0]
    assert adjust(x, [], 0, bias=[(3, 1.0), (3, 4.0)], temp=2.0).tolist() == [1.0, -1.0, 0.5, 2.0]
    assert adjust(x, [9, -1], 0, rho=3.0).tolist() == x                       # ids outside the vocabulary
    z = adjust(x, [], 0, mask=np.array([False, True, True, False]))
    assert pick(z) == 2 and softmax(z)[0] == 0 and abs(softmax(z).sum() - 1) < 1e-15
    assert pick(adjust(x, [], 0, mask=np.zeros(4, bool))) == -1 and softmax(np.full(4, -np.inf)).tolist() == [0.0] * 4
    assert pick(np.array([1.0, 3.0, 3.0])) == 1
    assert pack(np.array([[True] + [False] * 31 + [True, True]])).tolist() == [[1, 3]]
