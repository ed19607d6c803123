"""The largest extents of the sequence operators' C ABI (no GPU: refusals come
before anything is launched, and workspaces are arithmetic)."""
import pytest

from paper_2101_09808_amd import conv as B
from tests.test_seq_abi import FAKE, NORMS, call, conv, norm, scan


@pytest.mark.parametrize("D", [(1 << 30) + 1, (1 << 31) - 1])
def test_channels_past_a_workgroups_32_bits(D):
    """A channel's index plus those of a workgroup has to stay in 32 bits."""
    p = norm(N=1, D=D, L=1, sum=FAKE, dout=FAKE, dx=FAKE, dweight=FAKE)
    for fn in ("seq_norm_fwd_workspace", "seq_norm_bwd_workspace"):
        assert call(fn, p, True) == B.CONV_ERANGE
    s = scan(N=1, D=D, L=1, S=1, G=1, checkpoints=None, initial_state=FAKE, final_state=FAKE)
    for fn in ("seq_selective_scan_fwd_workspace", "seq_selective_scan_bwd_workspace"):
        assert call(fn, s, True) == B.CONV_ERANGE


def test_the_largest_extents_are_taken():
    big = dict(N=1, D=1 << 30, L=1)
    for fn in ("seq_norm_fwd_workspace", "seq_norm_bwd_workspace"):
        assert call(fn, norm(**big), True) >= 0
    assert call("seq_selective_scan_bwd_workspace", scan(**big, S=1, G=1), True) > 0
    assert call("seq_causal_conv_bwd_workspace", conv(N=1, D=(1 << 31) - 1, L=1), True) == 0


def test_refused_before_the_launch():
    s = dict(N=1, D=(1 << 30) + 1, L=1, S=1, G=1, checkpoints=None, initial_state=FAKE, final_state=FAKE)
    for fn in ("seq_selective_scan_fwd", "seq_selective_scan_step"):
        assert call(fn, scan(**s)) == B.CONV_ERANGE
    for fn in NORMS:
        kw = dict(sum=FAKE, out=None) if fn.endswith("pre_bwd") else {}
        assert call(fn, norm(**{**dict(N=1, D=(1 << 30) + 1, L=1), **kw})) == B.CONV_ERANGE
