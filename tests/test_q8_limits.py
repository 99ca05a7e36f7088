"""The 8-bit integer layers at the edges of what they take: refusals and checks of overlap with rows in them (CPU; no call gets as far as a launch)."""
import ctypes as C
import random

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


def _overlap(x, x_stride, rows, width, codes, codes_stride):
    """Whether dlm_add_norm_q8 refuses codes beside bf16 rows for their overlap.  (Without a gain, which is asked for next, no call is launched.)"""
    assert api.lib().dlm_add_norm_q8(x, x_stride, rows, width, 1, None, 0, None, 0, 0, None, 1e-5, codes, codes_stride, T, None) == EINVAL
    assert "overlap" in _err() or "null argument" in _err(), _err()
    return "overlap" in _err()


def test_codes_beside_their_source_with_rows():
    """200 bf16 values (400 bytes) and 200 codes side by side in rows of 640 bytes: columns of one matrix of different widths."""
    for rows in (1, 2, 4, 1000):
        at = lambda d: _overlap(P, 320, rows, 200, P + d, 640)  # noqa: E731
        assert not at(400) and not at(432) and not at(-208) and not at(-240)
        assert at(384) and at(0) and at(-192) and at(-16)
        assert at(448) == (rows > 1) and at(640) == (rows > 1) and not at(640 * rows) and at(640 * (rows - 1))  # (the next row's values; behind the last)


def test_overlap_is_what_enumeration_says():
    rng = random.Random(7)
    said = {True: 0, False: 0}
    for _ in range(4000):
        rows, width = rng.randint(1, 6), rng.randint(1, 40)
        xs = -(-2 * width // 16) * 16 + 16 * rng.randint(0, 5)  # bytes
        cs = xs if rng.random() < 0.7 else -(-width // 16) * 16 + 16 * rng.randint(0, 8)
        if cs < width:
            continue
        d = 16 * rng.randint(-rows * max(xs, cs) // 16 - 3, rows * max(xs, cs) // 16 + 3)
        mine = {r * xs + i for r in range(rows) for i in range(2 * width)}
        theirs = {d + r * cs + i for r in range(rows) for i in range(width)}
        got = _overlap(P, xs // 2, rows, width, P + d, cs)
        if xs == cs:
            assert got == bool(mine & theirs), (rows, width, xs, cs, d)
        else:  # of different strides: refused where their spans meet
            assert got == (min(theirs) <= max(mine) and min(mine) <= max(theirs)), (rows, width, xs, cs, d)
        said[got] += 1
    assert min(said.values()) > 500
