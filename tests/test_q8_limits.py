"""The 8-bit integer layers at the edges of what they take: refusals and checks of overlap with rows in them (CPU; no call gets as far as a launch)."""
import ctypes as C

import pytest

from paper_2604_15750_amd import api

EINVAL, ECAPACITY = -1, -3
P = 1 << 44  # pointers that are never dereferenced, 2^42 bytes apart
Q, R, S, T = (P + (i << 42) for i in range(1, 5))


def _err():
    return api.lib().dlm_last_error().decode()


@pytest.mark.parametrize("rows,n,k", [(114528, 4794144, 96), (1 << 20, 524286, 256), (16384, 1 << 24, 96), (1 << 20, 1 << 18, 64)])
@pytest.mark.parametrize("gated", [0, 1])
def test_a_product_fits_one_launch(rows, n, k, gated):
    """Of 2^38 outputs at most, and of less than 2^32 threads: what is more is refused before anything is asked of the GPU."""
    plan = api.plan_q8_gemm(rows, n, k, gated)
    outputs, threads = n // 2 if gated else n, (plan["workgroups"] + 7) // 8 * 8 * (512 if plan["kernel"] == "tiled" else 2 * plan["cols"])
    if outputs * rows <= 1 << 38 and threads < 1 << 32:
        return  # (such a call would be launched)
    stride = -(-outputs // 8) * 8
    assert api.lib().dlm_q8_gemm(C.byref(api.dlm_q8_weight(n, k, gated, T)), P, k, Q, rows, R, stride, 1, None, 0, None) == ECAPACITY
    assert "launch" in _err()


def test_one_of_those_has_too_many_threads_alone():
    rows, n, k = 114528, 4794144, 96
    plan = api.plan_q8_gemm(rows, n, k, True)
    assert rows * n // 2 <= 1 << 38 and plan["workgroups"] * 512 >= 1 << 32
