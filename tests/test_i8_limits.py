"""Numbers of rows, channels and sequences next to 2^31, beyond which the kernels' indexes would not fit: refused before any launch, without a GPU."""
import ctypes as C

import pytest

from test_i8_abi import CACHED, PRODUCTS, _calls, lib  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("over,calls", [
    (dict(N=2 ** 30 + 1, ldy=2 ** 31 - 1), PRODUCTS), (dict(N=2 ** 31 - 1, ldy=2 ** 31 - 1), PRODUCTS),
    (dict(M=2 ** 30 + 1), ("gemm",)), (dict(M=2 ** 31 - 1), ("gemm",)),
    (dict(S=2 ** 30 + 1), CACHED), (dict(S=2 ** 31 - 1), CACHED)])
def test_numbers_beyond_2_to_the_30_are_refused(lib, over, calls):  # noqa: F811
    from paper_2511_11248_b200 import binding as B
    table = _calls(B, **over)
    for name in calls:
        with pytest.raises(B.TmanError) as e:
            table[name]()
        assert e.value.status == 2, name


def test_sizes_of_scratch_say_so_too(lib):  # noqa: F811
    out = C.c_size_t(0)
    assert lib.tman_workspace_bytes_i8(1, 2 ** 30 + 1, 64, 8, C.byref(out)) == 2 and lib.tman_workspace_bytes_i8(1, 8, 64, 2 ** 30 + 1, C.byref(out)) == 2
    assert lib.tman_workspace_bytes_i8(1, 2 ** 30, 64, 2 ** 30, C.byref(out)) == 0
