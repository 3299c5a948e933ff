"""The most elements that clipping takes: what its workspace functions answer is
what its calls refuse.  No kernel is launched and no pointer is followed."""
import ctypes

import pytest

MOST = (1 << 36) - 1


def _lib():
    import paper_2211_06934_amd as P
    return P.diffopt._lib


def _at(i):
    return ctypes.c_void_p(i << 40)


@pytest.mark.parametrize("n", [MOST + 1, 1 << 37, (1 << 37) + 1, 1 << 40, 1 << 62])
def test_beyond(n):
    import paper_2211_06934_amd as P
    lib = _lib()
    assert lib.diffopt_clip_norm_workspace(n) == -1
    assert lib.diffopt_clip_norm_fwd(_at(1), n, 1.0, 1e-6, _at(2), _at(3), _at(4), 4096, None) == -1 and "too many elements" in P.last_error()
    assert lib.diffopt_clip_norm_bwd(_at(1), None, _at(2), _at(3), n, 1e-6, _at(5), _at(4), 4096, None) == -1 and "too many elements" in P.last_error()
    with pytest.raises(ValueError):
        P.clip_norm_workspace(n)


def test_the_most():
    import paper_2211_06934_amd as P
    lib = _lib()
    need = lib.diffopt_clip_norm_workspace(MOST)
    assert 0 < need <= 1 << 16
    # the size is taken: the workspace is what is refused
    assert lib.diffopt_clip_norm_fwd(_at(1), MOST, 1.0, 1e-6, _at(2), _at(3), _at(4), need - 1, None) == -1 and "workspace" in P.last_error()
