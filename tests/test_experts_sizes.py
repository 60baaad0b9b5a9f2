"""Sizes that the calls on sorted tokens refuse (no GPU needed: nothing is launched)."""
import ctypes as C

import pytest

P = 1 << 20   # an address that is never followed


@pytest.mark.parametrize("H", [2 ** 31 - 1, 2 ** 31 - 65535])
def test_rows_at_the_end_of_the_32_bit_counts(H):
    from paper_2401_13920_b200 import binding as B
    for dt in (B.BF16, B.F32):
        s = C.byref(B.Shape(1, H, 1, 1, 1, dt, 0))
        assert B._lib.locmoe_sort(s, 1, P, P, P, P, P, P, P, None) == -7
        assert B._lib.locmoe_unsort(s, 1, P, P, P, P, P, None) == -7
        assert B._lib.locmoe_unsort_grad(s, 1, P, P, P, P, P, P, P, None) == -7
        g = B.SortGrad(dxs=P, slot=P, dx=P)
        assert B._lib.locmoe_sort_grad(s, 1, C.byref(g), None, 0, None) == -7
