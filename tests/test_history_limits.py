"""The largest sizes that the history attention takes and the first that it refuses (no GPU: the
calls that pass every check end at the launch)."""

import ctypes

from paper_2607_27744_amd import _lib
from test_history_abi import _packed, _paged, lib, no_gpu   # noqa: F401 (lib: a fixture)

NO_LAUNCH = 4                             # ROCS_ERR_HIP: there is no device
TOP = 2 ** 31 - 4096


def _at(address):
    return ctypes.c_void_p(address)       # never dereferenced, far from the other arrays


@no_gpu
def test_keys_stay_clear_of_32_bits(lib):   # noqa: F811
    # The kernels' key indices pass a history's end by less than 4,096.
    kw = dict(H=1, Hk=1, D=1, N=1, R=1, most=64, k=_at(2 ** 40), v=_at(2 ** 41))
    for rows, status in ((TOP, NO_LAUNCH), (TOP + 1, _lib.UNSUPPORTED), (2 ** 31 - 1, _lib.UNSUPPORTED),
                         (2 ** 31, _lib.UNSUPPORTED)):
        assert _packed(lib, L=rows, **kw) == status
    kw = dict(H=1, Hk=1, D=1, N=1, R=1, S=1, most=64, table=_at(2 ** 40))
    for width, page, status in ((TOP, 1, NO_LAUNCH), (TOP + 1, 1, _lib.UNSUPPORTED),
                                (2 ** 27 - 256, 16, NO_LAUNCH), (2 ** 27 - 1, 16, _lib.UNSUPPORTED)):
        assert _paged(lib, W=width, page=page, **kw) == status


@no_gpu
def test_workgroups_of_one_launch(lib):   # noqa: F811
    kw = dict(H=1, Hk=1, D=1, dtype=0, L=64, most=64, R=1, q=_at(2 ** 40), out=_at(2 ** 41))
    assert _packed(lib, N=2 ** 28 - 64, **kw) == NO_LAUNCH
    assert _packed(lib, N=2 ** 28, **kw) == _lib.UNSUPPORTED

