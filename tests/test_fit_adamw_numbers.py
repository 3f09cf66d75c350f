"""AdamW: numbers at the ends of what 32 bits hold."""
import ctypes as C

import pytest

from paper_2206_05279_amd import binding as pb

P = 1 << 20          # an address that nothing follows: these calls are refused


@pytest.mark.parametrize("bad", [dict(lr=1e39), dict(eps=1e300), dict(grad_scale=-1e39), dict(lr=1e38, mult=100.0), dict(lr=1e20, decay=1e20),
                                 dict(lr=1e38, beta1=0.99999)])
def test_what_32_bits_do_not_hold_is_refused(bad):
    k = dict(lr=1e-3, eps=1e-8, grad_scale=1.0, mult=1.0, decay=0.0, beta1=0.9)
    k.update(bad)
    par = pb.pilc_adamw_params(k["lr"], k["beta1"], 0.999, k["eps"], k["grad_scale"], 1, 0, 0, 32, 0)
    t = (pb.pilc_adamw_tensor * 1)(pb.pilc_adamw_tensor(P, P, P, P, None, None, 10, k["mult"], k["decay"]))
    assert pb.lib().pilc_adamw_step(C.byref(par), t, 1, None) == pb.PILC_E_ARG
