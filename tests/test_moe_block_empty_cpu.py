"""The norms' forward call on no tokens, where empty tensors have no address: nothing to do and nothing refused, but for what is
wrong with any number of tokens.  (The gradient call writes sums over no tokens; the GPU tests have it.)"""
import ctypes

import pytest

from paper_2604_02715_amd import binding as B

P = 1 << 20                     # stands for a device address; no accepted call reaches it


def norm(flags=0, y=None, residual=None, gate=None, w_post=None, w_pre=P, out=None, n=None, **kw):
    fields = dict(hidden=64, y_type=B.F32, residual_type=B.BF16, weight_type=B.BF16, flags=flags, eps=1e-6, scale=1.0)
    B.fluxmoe_block_norm(ctypes.pointer(B.NormDesc(**dict(fields, **kw))), 0, y, residual, gate, w_post, w_pre, out, n)


@pytest.mark.parametrize("kw", [dict(), dict(w_post=P), dict(flags=B.NORM_GATE_TOKEN), dict(flags=B.NORM_GATE_TOKEN, gate=P), dict(w_post=P, y=P),
                                dict(flags=B.NORM_GATE_CHANNEL, gate=P), dict(flags=B.NORM_GATE_TOKEN | B.NORM_GATE_SIGMOID, w_post=P)])
def test_no_tokens_is_no_work(kw):
    norm(**kw)


@pytest.mark.parametrize("kw", [dict(flags=B.NORM_GATE_CHANNEL), dict(gate=P), dict(flags=B.NORM_GATE_SIGMOID), dict(flags=3), dict(hidden=0), dict(y_type=2),
                                dict(y_stride=63), dict(w_post=P + 1), dict(flags=B.NORM_GATE_CHANNEL, gate=P + 2)])
def test_what_is_refused_all_the_same(kw):
    with pytest.raises(B.FluxmoeError) as e:
        norm(**kw)
    assert e.value.status == -1
