"""Results of the operators that lie on operands, or on one another, where an entry
point does not allow it: refused before any device call.  No pointer is followed."""
import ctypes

import pytest

from test_host_operators import BF16, F32, _binding, _refused


def _p(at):
    return ctypes.c_void_p(at)


def _h(at, b=1024, t=64, h=8):
    return ctypes.byref(_binding()[2](at, b, t, h))


def _fwd(q=0x10000, k=0x20000, v=0x30000, out=0x40000, state=None, state_out=None, dtype=F32):
    lib, _, _ = _binding()
    return lib.diffopt_linattn_fwd(_h(q), _h(k), _h(v), _p(64), None, _p(state), 2, 9, 4, 2, 8, 8, dtype, 1.0, _h(out), _p(state_out), None, 0, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_linattn_fwd_out_is_no_operand(name, dtype):
    _refused(_fwd(**{name: 0x40000}, dtype=dtype), "must not be an operand")


@pytest.mark.parametrize("shift", [4, 512, 2 * 2 * 8 * 8 * 4 - 4])
@pytest.mark.parametrize("sign", [-1, 1])
def test_linattn_fwd_states_are_one_or_apart(shift, sign):
    _refused(_fwd(state=0x50000, state_out=0x50000 + sign * shift), "state_out must be state or lie apart")


def _bwd(dq=0x50000, dk=0x60000, dv=0x70000, dout=0x40000, state=None, ds1=None, ds=None):
    lib, _, _ = _binding()
    return lib.diffopt_linattn_bwd(_h(dout), _p(ds1), _h(0x10000), _h(0x20000), _h(0x30000), _p(64), None, _p(state), 2, 9, 4, 2, 8, 8, F32, 1.0,
                                   _h(dq), _h(dk), _h(dv), _p(ds), None, 0, None)


@pytest.mark.parametrize("result", ["dq", "dk", "dv"])
@pytest.mark.parametrize("operand", [0x10000, 0x20000, 0x30000, 0x40000])
def test_linattn_bwd_results_are_no_operands(result, operand):
    _refused(_bwd(**{result: operand}), "must not be an operand")


def test_linattn_bwd_results_are_apart():
    _refused(_bwd(dq=0x60000), "two results")
    _refused(_bwd(dv=0x60000), "two results")
    _refused(_bwd(dv=0x50000), "two results")
    for shift in (-4, 0, 4):
        _refused(_bwd(state=0x80000, ds=0x80000 + shift), "dstate must")
        _refused(_bwd(ds1=0x80000, ds=0x80000 + shift), "dstate must")


@pytest.mark.parametrize("operand", [0x10000, 0x20000, 0x30000])
def test_linattn_step_out_is_no_operand(operand):
    lib, _, _ = _binding()
    rc = lib.diffopt_linattn_step(_h(0x10000), _h(0x20000), _h(0x30000), _p(64), 2, 4, 2, 8, 8, F32, 1.0, _p(0x80000), _h(operand), None)
    _refused(rc, "must not be an operand")
