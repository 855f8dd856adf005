"""Calls behind a prompt that the general tests do not make: refusals on the host, before anything is launched."""
import pytest

import test_host_onward as base
from paper_2603_00198_amd import binding
from test_host_onward import BF16, EHIP, EUNSUPPORTED, P, _i32, _seqs


def _call(name, **at):
    args = list(base._cases()[name][0])
    for k, v in at.items():
        args[int(k[1:])] = v
    return getattr(binding.lib(), name)(*args)


def test_more_threads_than_a_launch_has_are_refused():
    """A launch counts its threads in 32 bits: sizes beyond that are refused with STRD_EUNSUPPORTED, the last below it goes on (to the GPU that is not there)."""
    base._no_gpu()
    far = 1 << 60
    rope = dict(_0=P, _2=far, _4=1, _9=0, _1=512, _3=512)
    assert _call("strd_rope", _12=1 << 25, **rope) == EHIP and _call("strd_rope", _12=(1 << 25) + 1, **rope) == EUNSUPPORTED
    # heads times nodes: a workgroup each in the join
    assert _call("strd_attn_tree_step", _8=64, _9=1 << 15, _18=1 << 62) == EHIP
    assert _call("strd_attn_tree_step", _8=64, _9=(1 << 15) + 2, _18=1 << 62) == EUNSUPPORTED
    # a channel at a time, since the pitch is odd: 2^30 rows of 33 channels, eight rows to a thread
    conv = dict(_1=33, _4=None, _5=None, _10=1, _14=33, _15=0)
    assert _call("strd_conv1d_silu_varlen", _9=_seqs((1 << 29, 0)), **conv) == EHIP
    assert _call("strd_conv1d_silu_varlen", _9=_seqs((1 << 30, 0)), **conv) == EUNSUPPORTED
