"""Sizes at which 32-bit positions, channels or launches of the operators around the recurrence would overflow: refused
by the C entry points before any launch (fake, never dereferenced, aligned pointers are used)."""
import pytest

from paper_2606_08804_amd import mixer

FAKE = 1 << 20
OK, EINVAL, EUNSUPPORTED, ENOWORKSPACE = range(4)
LONGEST = (1 << 31) - 64


def conv_fwd(N=1, T=1, D=1, W=4, cu=None):
    return mixer.lib().qdelta_conv_fwd(N, T, cu, D, W, 1, 1, FAKE, D, FAKE, None, None, FAKE, None, None)


def conv_bwd(N=1, T=1, D=1, W=4, cu=None, ws=1 << 60, dw=FAKE, db=None):
    return mixer.lib().qdelta_conv_bwd(N, T, cu, D, W, 1, 1, FAKE, D, FAKE, None, None, FAKE, None, FAKE, dw, db, None, FAKE,
                                       ws, None)


def scan(fn, T, cu=None, ws=1 << 60):
    return fn(1, T, cu, 1, 1, 1, 1, 1, 1, FAKE, 1, FAKE, FAKE, FAKE, 1, FAKE, 1, None, None, None,
              *((FAKE, None) if fn is mixer.lib().qdelta_scan_fwd else (FAKE, None) + (FAKE,) * 5 + (None,) * 3), FAKE, ws, None)


@pytest.mark.parametrize("cu", [None, FAKE])
@pytest.mark.parametrize("T", [LONGEST + 1, (1 << 31) - 33, (1 << 31) - 1])
def test_positions_past_32_bits_are_refused(T, cu):
    """A tile that starts near token 2^31 would end past it: its end would be negative."""
    L = mixer.lib()
    assert conv_fwd(T=T, cu=cu) == conv_bwd(T=T, cu=cu) == EUNSUPPORTED
    assert scan(L.qdelta_scan_fwd, T, cu) == scan(L.qdelta_scan_bwd, T, cu) == EUNSUPPORTED
    assert mixer.conv_workspace_bytes(1, T, 1, 4, packed=cu is not None) == 0
    assert mixer.scan_workspace_bytes(1, T, 1, 1, 1, 1, packed=cu is not None, is_bwd=True) == 0


@pytest.mark.parametrize("cu", [None, FAKE])
def test_the_longest_sequence_is_taken(cu):
    """As far as its workspace; the scan has at most 2^23 - 9 chunks of 64 tokens."""
    L = mixer.lib()
    assert conv_bwd(T=LONGEST, cu=cu, ws=0) == ENOWORKSPACE and mixer.conv_workspace_bytes(1, LONGEST, 1, 4, cu is not None)
    longest = ((1 << 23) - 10) * 64
    for fn, back in ((L.qdelta_scan_fwd, False), (L.qdelta_scan_bwd, True)):
        assert scan(fn, longest, cu, ws=0) == ENOWORKSPACE and scan(fn, 1 << 29, cu) == EUNSUPPORTED
        assert mixer.scan_workspace_bytes(1, longest, 1, 1, 1, 1, cu is not None, back)


def test_channels_past_32_bits_or_a_launch_are_refused():
    """The taps of 2^29 channels are 2^31 values; the weight's gradient of 2^26 is summed by 16 threads for each of 5 x
    2^26 columns, which would fail after the other gradients have been launched."""
    step = lambda D, W: mixer.lib().qdelta_conv_step(1, D, W, 1, 1, FAKE, D, FAKE, None, FAKE, FAKE, FAKE, None)     # noqa: E731
    for D, W in (((1 << 29) + 1, 4), (1 << 29, 4), (1 << 30, 2)):
        assert conv_fwd(D=D, W=W) == conv_bwd(D=D, W=W) == step(D, W) == EUNSUPPORTED, (D, W)
        assert mixer.conv_workspace_bytes(1, 1, D, W) == 0
    assert conv_bwd(D=1 << 26) == conv_bwd(D=1 << 26, dw=None, db=FAKE) == EUNSUPPORTED
    assert conv_bwd(D=(1 << 29) - 1, ws=0) == ENOWORKSPACE
