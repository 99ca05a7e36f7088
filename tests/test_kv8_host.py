"""Host-only checks of the 8-bit cache's entry points: shapes, sizes and refusals (no call gets as far as the GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_15750_amd import api

EINVAL, ESHAPE, ECAPACITY = -1, -2, -3
P = 1 << 40  # a pointer that is never dereferenced: validation fails first


def _ints(*v):
    return (C.c_int32 * len(v))(*v)


def _err():
    return api.lib().dlm_last_error().decode()


def _cache(slots=4, max_len=100, n_kv=2, hd=64, fmt=0, data=P):
    return C.byref(api.dlm_kv8_cache(slots, max_len, n_kv, hd, fmt, data))


def test_cache_bytes():
    f = api.lib().dlm_kv8_bytes
    assert C.sizeof(api.dlm_kv8_cache) == 32
    # blocks of 32 positions: 2 x 32 x hd codes and 64 scales
    assert f(1, 1, 1, 32) == 64 * 32 + 64 and f(3, 33, 2, 128) == 3 * 2 * 2 * (64 * 128 + 64)
    assert f(1000, 1 << 20, 32, 128) == 1000 * 32 * (1 << 15) * (64 * 128 + 64)  # (beyond 32 bits)
    for bad in ((0, 1, 1, 32), (1, 0, 1, 32), (1, 1, 0, 32), (1, 1, 1, 48), (1, 1, 65536, 32), (-1, 1, 1, 32), (2**31 - 1, 2**31 - 1, 65535, 128)):
        assert f(*bad) == 0, bad


@pytest.mark.parametrize("name", ["dlm_kv8_write", "dlm_kv8_read"])
def test_span_refusals(name):
    f = getattr(api.lib(), name)

    def call(c=None, k=P, v=P, stride=128, dtype=1, off=_ints(0, 3), start=_ints(5), slot=None, n=1):
        return f(c or _cache(), k, v, stride, dtype, off, start, slot, n, None)

    assert call(k=None) == EINVAL and call(v=None) == EINVAL and call(off=None) == EINVAL and call(start=None) == EINVAL and "null" in _err()
    assert f(None, P, P, 128, 1, _ints(0, 3), _ints(5), None, 1, None) == EINVAL and call(_cache(data=None)) == EINVAL
    assert call(_cache(data=P + 8)) == EINVAL and call(k=P + 2) == EINVAL and call(v=P + 8) == EINVAL and "aligned" in _err()
    assert call(_cache(fmt=2)) == EINVAL and call(dtype=2) == EINVAL
    assert call(stride=127) == EINVAL and call(stride=120) == EINVAL and call(stride=130) == EINVAL and call(stride=130, dtype=0) == EINVAL and call(stride=-128) == EINVAL
    for c in (_cache(slots=0), _cache(max_len=0), _cache(n_kv=0), _cache(hd=96)):
        assert call(c) == ESHAPE
    assert call(n=0) == EINVAL and call(n=33) == ECAPACITY
    assert call(off=_ints(1, 3)) == EINVAL and call(off=_ints(0, -1)) == EINVAL
    assert call(slot=_ints(4)) == EINVAL and call(slot=_ints(-1)) == EINVAL and "slot" in _err()
    assert call(start=_ints(-1)) == EINVAL and call(start=_ints(98)) == ECAPACITY and call(off=_ints(0, 96)) == ECAPACITY
    assert call(start=_ints(2**31 - 1)) == ECAPACITY
    # nothing to do: no launch
    assert call(off=_ints(0, 0), start=_ints(100)) == 0
    if name == "dlm_kv8_write":
        assert call(off=_ints(0, 1, 2), start=_ints(0, 50), slot=_ints(1, 1), n=2) == EINVAL and "twice" in _err()


def test_attention_refusals():
    f = api.lib().dlm_kv8_attention
    need = api.lib().dlm_kv8_attention_workspace(3, 4, 64)
    assert need > 0 and api.lib().dlm_kv8_attention_workspace(0, 4, 64) == 0 and api.lib().dlm_kv8_attention_workspace(3, 4, 65) == 0

    def call(c=None, q=P, stride=256, out=2 * P, dtype=1, n_q=4, off=_ints(0, 3), keys=_ints(7), slot=None, n=1, mask=None, words=0, ws=3 * P, size=need):
        return f(c or _cache(), q, stride, out, dtype, n_q, off, keys, slot, n, mask, words, ws, size, None)

    assert call(q=None) == EINVAL and call(out=None) == EINVAL and call(off=None) == EINVAL and call(keys=None) == EINVAL
    assert call(_cache(data=None)) == EINVAL and call(_cache(fmt=-1)) == EINVAL and call(dtype=3) == EINVAL
    assert call(_cache(hd=16)) == ESHAPE and call(n_q=3) == ESHAPE and call(n_q=0) == ESHAPE and call(n_q=65536) == ESHAPE
    assert call(q=P + 2) == EINVAL and call(out=2 * P + 4) == EINVAL and call(ws=3 * P + 4) == EINVAL and call(mask=P + 2, words=1) == EINVAL
    assert call(stride=252) == EINVAL and call(stride=255) == EINVAL and call(stride=260, dtype=1) == EINVAL
    assert call(out=P) == EINVAL and call(out=P + 1024) == EINVAL and call(out=P - 1024) == EINVAL and "overlaps" in _err()
    assert call(n=0) == EINVAL and call(n=33) == ECAPACITY and call(off=_ints(0, -3)) == EINVAL and call(off=_ints(2, 3)) == EINVAL
    assert call(slot=_ints(4)) == EINVAL
    assert call(keys=_ints(-1)) == EINVAL and call(keys=_ints(101)) == ECAPACITY
    assert call(mask=P, words=0) == EINVAL and call(mask=P, words=1, keys=_ints(2)) == EINVAL
    assert call(mask=P, words=1, off=_ints(0, 33), keys=_ints(50)) == ECAPACITY and "mask_words" in _err()
    assert call(size=need - 1) == ECAPACITY and call(ws=None) == ECAPACITY and "workspace" in _err()
    assert call(off=_ints(0, 0), size=0, ws=None) == 0  # nothing to do


def test_norm_rope_refusals():
    f = api.lib().dlm_qk_norm_rope

    def call(x=P, xs=512, rows=3, n_q=4, n_kv=2, hd=64, dtype=1, gq=P, gk=P, eps=1e-5, theta=1e4, pos=P, out=2 * P, os=384):
        return f(x, xs, rows, n_q, n_kv, hd, dtype, gq, gk, eps, theta, pos, out, os, None)

    assert call(x=None) == EINVAL and call(out=None) == EINVAL and call(pos=None) == EINVAL
    assert call(dtype=2) == EINVAL and call(hd=80) == ESHAPE
    assert call(rows=-1) == ESHAPE and call(n_q=-1) == ESHAPE and call(n_q=0, n_kv=0) == ESHAPE and call(n_q=65535) == ESHAPE and call(n_q=2**31 - 1, n_kv=2**31 - 1) == ESHAPE
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert call(eps=bad) == EINVAL and call(theta=bad) == EINVAL, bad
    assert call(x=P + 8) == EINVAL and call(out=2 * P + 2) == EINVAL and call(gq=P + 4) == EINVAL and call(gk=P + 4) == EINVAL and call(pos=P + 2) == EINVAL
    assert call(xs=383) == EINVAL and call(xs=380) == EINVAL and call(os=386) == EINVAL
    assert call(out=P, os=384) == EINVAL and call(out=P + 16, os=512) == EINVAL and "overlaps" in _err()  # (in place only with the same stride)
    assert call(rows=0, gq=None, gk=None) == 0


def test_python_refusals_before_the_library():
    """What a C call cannot see: tensors elsewhere, of other types, shapes or orders, lists that are too short or no 32-bit integers."""
    c = object.__new__(api.Kv8Cache)
    c.slots, c.max_len, c.n_kv, c.head_dim = 2, 64, 2, 64
    c.data = torch.zeros(16, dtype=torch.uint8)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: api.dlm_kv8_write(c, x, x, [0, 4], [0]), lambda: api.dlm_kv8_read(c, [0, 4], [0], k=x, v=x),
                 lambda: api.dlm_kv8_attention(c, x, [0, 4], [4]), lambda: api.dlm_qk_norm_rope(x[:, 0], torch.zeros(4, dtype=torch.int32), 1, 0, 64)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    for bad in ([2**31], [-2**31 - 1], [1.5], ["1"]):
        with pytest.raises(ValueError):
            api._int32s("start", bad, 1)
    with pytest.raises(ValueError):
        api._int32s("start", [1], 2)
    assert api._int32s("slot", None, 3) is None and api._int32s("start", torch.tensor([1, 2]), 2) == bytes((C.c_int32 * 2)(1, 2))
    with pytest.raises(ValueError):
        api.Kv8Cache(1, 64, 2, 64, format="e5m2", device="cpu")
    with pytest.raises(api.DlmError, match="ESHAPE"):
        api.Kv8Cache(1, 64, 2, 65, device="cpu")
