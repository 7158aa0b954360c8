"""The factor of the AdamW step's gradients is read while the step writes: it may lie in no buffer that is written.  No GPU: refusals come before the first launch."""
import ctypes as C

import pytest

from paper_2308_10087_amd.binding import gnntrain_adamw_tensor, lib

BUF = (C.c_char * (1 << 16))()
AT = (C.addressof(BUF) + 255) // 256 * 256  # never read


def _refused(scale, bits):
    t = gnntrain_adamw_tensor()
    for name, x in dict(p=AT, g=AT + 1000, m=AT + 2000, v=AT + 3000, m_scale=AT + 4096, v_scale=AT + 4200, compute=AT + 5000, compute_dtype=1, count=100, weight_decay=0.1).items():
        setattr(t, name, x)
    # (a list that is refused anyway, for its second tensor's sake: what is told is told of the first fault)
    bad = gnntrain_adamw_tensor()
    bad.count = -1
    both = (gnntrain_adamw_tensor * 2)(t, bad)
    assert lib.gnntrain_adamw_step(both, 2, bits, 1e-3, 0.9, 0.999, 1e-8, scale, 1, 0, None) == -1
    assert "count" in lib.gnntrain_last_error(None).decode()
    rc = lib.gnntrain_adamw_step((gnntrain_adamw_tensor * 1)(t), 1, bits, 1e-3, 0.9, 0.999, 1e-8, scale, 1, 0, None)
    return rc == -1 and "grad_scale" in lib.gnntrain_last_error(None).decode()


@pytest.mark.parametrize("scale", [0, 396, 2000, 3096, 5000, 5196])
def test_a_factor_among_what_is_written_is_refused(scale):
    assert _refused(AT + scale, 8)


@pytest.mark.parametrize("scale", [2396, 3396])
def test_fp32_states_reach_further(scale):
    assert _refused(AT + scale, 32)


@pytest.mark.parametrize("scale", [4096, 4200])
def test_the_factors_of_blocks_too(scale):
    assert _refused(AT + scale, 8)


@pytest.mark.parametrize("off", [1, 2])
def test_its_alignment(off):
    assert _refused(AT + 6000 + off, 8)
