"""Refusals of the rotary positions at the C entries, on the CPU: outputs that hold a row
more than once, and frequencies whose base is past fp64."""
import ctypes

import pytest

from paper_2608_02474_amd import _lib, api

FAKE, FAKE2 = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x20000)
F3, F4 = ctypes.c_void_p(0x30000), ctypes.c_void_p(0x40000)


def _cfg(B, L, H, Hk, q, k, qo, ko):
    return _lib.RotaryCfg(B, L, H, Hk, 64, 64, _lib.ECHO_ROTARY_HALF, _lib.ECHO_BF16, 0, 0, 0, 0, 1.0, 0, _lib.Strides(*q),
                          _lib.Strides(*k), _lib.Strides(*qo), _lib.Strides(*ko))


@pytest.mark.parametrize("at", range(3))
def test_outputs_hold_no_row_twice(at):
    """In place over a repeated row too: it would be turned once for each time it is there."""
    lib = _lib.load()
    full = [5 * 2 * 64, 2 * 64, 64]
    zero = [0 if i == at else s for i, s in enumerate(full)]

    def run(B=3, L=5, H=2, Hk=2, q=full, k=full, qo=full, ko=full, out=F3, k_out=F4):
        return lib.echo_rotary(ctypes.byref(_cfg(B, L, H, Hk, q, k, qo, ko)), FAKE, FAKE2, None, FAKE, out, k_out, None)
    assert run(qo=zero) == _lib.ECHO_EINVAL
    assert run(ko=zero) == _lib.ECHO_EINVAL
    assert run(q=zero, qo=zero, out=FAKE) == _lib.ECHO_EINVAL
    assert run(k=zero, ko=zero, k_out=FAKE2) == _lib.ECHO_EINVAL
    assert run(B=0, qo=zero) == _lib.ECHO_OK                       # nothing to write


def test_bases_past_fp64_are_refused():
    """base factor^(dims / (dims - 2)) overflows: every frequency but the first would be 0."""
    kw = dict(scaling="base", base=1e300, factor=1e6)
    with pytest.raises(RuntimeError, match="echo_rotary_frequencies"):
        api.rotary_frequencies(4, **kw)
    freq, _, _ = api.rotary_frequencies(64, **{**kw, "base": 1e4})
    assert all(f > 0 for f in freq)
