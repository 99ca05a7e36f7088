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
    # keys that are shared between workgroups: a partial output, a maximum and a sum per share, row and head
    long = dict(c=_cache(max_len=5000), off=_ints(0, 1), keys=_ints(5000))
    assert call(ws=None, **long) == ECAPACITY and call(size=1000, **long) == ECAPACITY and "workspace" in _err()
    least = int(_err().split("<")[1])
    assert 1000 < least <= api.lib().dlm_kv8_attention_workspace(1, 4, 64) and least % (4 * 66 * 4) == 0 and call(size=least - 1, **long) == ECAPACITY
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


def test_launches_that_would_be_too_large():
    """A launch has fewer than 2^32 threads in a dimension, and its other dimensions at most 65535 workgroups."""
    L = api.lib()
    rows = 4 * ((1 << 24) - 1) + 1  # 4 rows a workgroup
    assert L.dlm_qk_norm_rope(P, 64, rows, 1, 0, 32, 1, None, None, 1e-5, 1e4, P, 2 * P, 64, None) == ECAPACITY and "too many rows" in _err()
    # blocks of 32 positions x heads
    n = 1 << 29
    big = _cache(slots=2, max_len=n, n_kv=1, hd=32)
    for f in (L.dlm_kv8_write, L.dlm_kv8_read):
        assert f(big, 2 * P, 3 * P, 32, 1, _ints(0, n), _ints(0), None, 1, None) == ECAPACITY and "too many rows" in _err()
        assert f(big, 2 * P, 3 * P, 32, 1, _ints(0, n // 2, n), _ints(0, 1), None, 2, None) == ECAPACITY
        assert f(big, 2 * P, 3 * P, 32, 1, _ints(0, n // 2, n // 2 + 1, 2**31 - 1), _ints(0, 1, 2), _ints(0, 1, 0), 3, None) == (EINVAL if f is L.dlm_kv8_write else ECAPACITY)
    # tiles of 32 queries of a kv head, of one sequence and of several
    rows = 32 * 65535 // 4 + 1
    for off, keys in ((_ints(0, rows), _ints(5)), (_ints(0, 1, rows), _ints(5, 7)), (_ints(0, 2**31 - 1), _ints(5))):
        assert L.dlm_kv8_attention(_cache(), 2 * P, 512, 9 * P, 1, 8, off, keys, None, len(keys), None, 0, None, 0, None) == ECAPACITY and "too many rows" in _err()
    # positions that a block's end would take past 31 bits
    assert L.dlm_kv8_bytes(1, 2**31 - 1, 1, 32) == 0 and L.dlm_kv8_bytes(1, 2**31 - 255, 1, 32) == 0 and L.dlm_kv8_bytes(1, 2**31 - 256, 1, 32) > 0


def test_overlaps():
    """Columns of one matrix share no byte; an output that shares one with what is read is refused.  (What is not refused ends at a row
    count that is: nothing is launched.)"""
    L, d = api.lib(), P  # the cache's memory
    f = L.dlm_kv8_read
    size = L.dlm_kv8_bytes(4, 100, 2, 64)

    def read(k, v, stride, rows=3, write=False):
        return (L.dlm_kv8_write if write else f)(_cache(), k, v, stride, 1, _ints(0, rows), _ints(0), None, 1, None)

    for stride, apart in ((128, 0), (128, 16), (128, 256 * 3 - 16), (400, 0), (400, 240), (400, 800 - 240), (400, 1600), (400, 1600 + 240), (400, 1600 - 240)):
        assert read(2 * P, 2 * P + apart, stride) == EINVAL and "overlaps v" in _err(), (stride, apart)
        assert read(2 * P + apart, 2 * P, stride) == EINVAL, (stride, apart)
    for k, v in ((d, 2 * P), (2 * P, d), (d + size - 16, 2 * P), (2 * P, d - 256), (d - 768 + 16, 2 * P)):
        for write in (False, True):
            assert read(k, v, 128, write=write) == EINVAL and "the cache" in _err(), (k - d, v - d)

    def attention(q=2 * P, out=3 * P, mask=4 * P, ws=5 * P, stride=256, off=_ints(0, 1), c=_cache(max_len=5000)):
        return L.dlm_kv8_attention(c, q, stride, out, 1, 4, off, _ints(5000), None, 1, mask, 4, ws, 1 << 30, None)

    for kw in (dict(out=d), dict(out=d - 496), dict(out=4 * P), dict(out=4 * P - 496), dict(out=2 * P + 496), dict(out=2 * P, stride=512), dict(ws=2 * P), dict(ws=3 * P + 496),
               dict(ws=4 * P), dict(ws=d), dict(q=d, ws=d)):
        assert attention(**kw) == EINVAL and "overlaps" in _err(), kw
    # rows and strides whose product passes 64 bits
    assert attention(out=2 * P + (1 << 45), stride=1 << 40, off=_ints(0, 100)) == EINVAL and "out overlaps q" in _err()

    def rope(x, out, xs, os, rows=3):
        return L.dlm_qk_norm_rope(x, xs, rows, 2, 0, 64, 1, None, None, 1e-5, 1e4, 6 * P, out, os, None)

    for x, out, xs, os in ((P, P + 16, 128, 128), (P, P + 240, 400, 400), (P, P + 800 - 240, 400, 400), (P, P + 256, 400, 408), (P, P, 400, 128), (P, P + 1600 + 240, 400, 400)):
        assert rope(x, out, xs, os) == EINVAL and "out overlaps x" in _err(), (out - x, xs, os)
        assert rope(out, x, os, xs) == EINVAL


def test_python_refusals_before_the_library(monkeypatch):
    """What a C call cannot see: tensors elsewhere, of other types, shapes or orders, lists that are too short or no 32-bit integers."""
    c = api.Kv8Cache(2, 64, 2, 64, device="cpu")
    monkeypatch.setattr(api, "_device", lambda: 0)
    monkeypatch.setattr(api, "_stream", lambda: 0)
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
    with pytest.raises(AttributeError):  # (the library has its address)
        c.data = torch.zeros_like(c.data)


def test_sizes_beyond_32_bits(monkeypatch):
    """They would arrive at the library as their low 32 bits."""
    for bad in ((2**32 + 1, 64, 2, 64), (1, 2**32 + 64, 2, 64), (1, 64, 2**32 + 2, 64), (1, 64, 2, 2**32 + 64)):
        with pytest.raises(api.DlmError, match="ESHAPE"):
            api.Kv8Cache(*bad, device="cpu")
    monkeypatch.setattr(api, "_device", lambda: -1)
    monkeypatch.setattr(api, "_stream", lambda: 0)
    monkeypatch.setattr(api, "_gpu_of", lambda name, t: -1)
    many = torch.zeros(1, 128, dtype=torch.bfloat16).expand(2**32 + 1, 128)
    with pytest.raises(ValueError):
        api.dlm_qk_norm_rope(many, torch.zeros(1, dtype=torch.int32).expand(2**32 + 1), 1, 1, 64, out=many)
    few = torch.zeros(3, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.dlm_qk_norm_rope(few, torch.zeros(3, dtype=torch.int32), 2**32 + 1, 1 - 2**32, 64)
    cache = api.Kv8Cache(2, 64, 2, 64, device="cpu")
    with pytest.raises(ValueError):  # fewer offsets than sequences
        api.dlm_kv8_read(cache, [0], [0])
    with pytest.raises(api.DlmError, match="EINVAL"):  # (the library's: offsets that decrease; a row so that it is asked)
        api.dlm_kv8_read(cache, [0, -3], [0], k=few.unflatten(1, (2, 64)), v=few.clone().unflatten(1, (2, 64)))


# ---- the extension and the way through ctypes: the same C call, or the same refusal ----------------------------------------------------

VP, I32, I64, F32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
SPAN = C.CFUNCTYPE(I32, VP, VP, VP, I64, I32, VP, VP, VP, I32, VP)
ATTENTION = C.CFUNCTYPE(I32, VP, VP, I64, VP, I32, I32, VP, VP, VP, I32, VP, I32, VP, C.c_size_t, VP)
ROPE = C.CFUNCTYPE(I32, VP, I64, I32, I32, I32, I32, I32, VP, VP, F32, F32, VP, VP, I64, VP)


@pytest.fixture
def both(monkeypatch):
    """both(f): what f's call hands to the library through the extension and through ctypes, or the exceptions' types; both.taken: whether
    the extension made the call itself.  CPU tensors stand for the GPU's (index -1); nothing is launched."""
    ext = api._kv8_calls()
    assert ext is not None, "the extension has not been built"
    L, seen = api.lib(), []
    ints = lambda p, n: None if not p else tuple((C.c_int32 * n).from_address(p))  # noqa: E731

    class Both:
        status = 0

        def __call__(self, f):
            out = []
            for through in (True, False):
                seen.clear()
                self.taken = False
                monkeypatch.setattr(api, "_kv8_calls", (lambda: Spy) if through else (lambda: None))
                try:
                    f()
                    out.append(list(seen))
                except Exception as e:  # noqa: BLE001
                    out.append(type(e))
                if through:
                    taken = self.taken
            self.taken = taken
            return out

    self = Both()

    def span(which):
        def call(c, k, v, stride, dt, off, start, slot, n, st):
            seen.append((which, c, k, v, stride, dt, ints(off, n + 1), ints(start, n), ints(slot, n), n, st))
            return self.status
        return SPAN(call)

    def attention(c, q, stride, out, dt, n_q, off, keys, slot, n, mask, words, ws, size, st):
        seen.append((c, q, stride, out, dt, n_q, ints(off, n + 1), ints(keys, n), ints(slot, n), n, mask, words, bool(ws), size, st))
        return self.status

    def rope(*a):
        seen.append(a)
        return self.status

    calls = [span(0), span(1), ATTENTION(attention), ROPE(rope)]

    class Recorder:
        dlm_kv8_write, dlm_kv8_read, dlm_kv8_attention, dlm_qk_norm_rope = calls
        dlm_kv8_attention_workspace, dlm_last_error = staticmethod(lambda *a: 0), L.dlm_last_error

    class Spy:
        @staticmethod
        def ask(f, args):
            rc = f(*args)
            self.taken = rc is not None
            assert self.taken == (len(seen) == 1)
            return rc

        span, attention, rope = (staticmethod(lambda *a, f=f: Spy.ask(f, a)) for f in (ext.span, ext.attention, ext.rope))

    real = [C.cast(f, VP).value for f in (L.dlm_kv8_write, L.dlm_kv8_read, L.dlm_kv8_attention, L.dlm_qk_norm_rope)]
    for name, value in (("lib", lambda: Recorder), ("_device", lambda: -1), ("_stream", lambda: 0x1230), ("_gpu_of", lambda name, t: -1)):
        monkeypatch.setattr(api, name, value)
    ext.bind(*(C.cast(f, VP).value for f in calls))
    yield self
    ext.bind(*real)


BF = torch.bfloat16
LISTS = [([0, 3, 5], [7, 2]), ((0, 3, 5), (7, 2)), ([0, 3, 5, 9], [7, 2]), (torch.tensor([0, 3, 5]), [7, 2]), ([0, 3, 5], [7.0, 2]), ([0, 3], [7, 2]),
         ([0, 3, 7], [7, 2]), ([0, 3, 5], [2**31, 2]), ([0, 3, 5], ["7", 2]), ([0] * 41, [0] * 40)]


@pytest.fixture(scope="module")
def cpu_cache():
    return api.Kv8Cache(50, 64, 2, 64, device="cpu")


@pytest.mark.parametrize("write", [True, False])
@pytest.mark.parametrize("off,start", LISTS)
def test_span_calls_either_way(both, cpu_cache, write, off, start):
    wide = torch.zeros(6, 400, dtype=BF)
    k, v = torch.zeros(6, 2, 64, dtype=BF), torch.ones(6, 2, 64, dtype=BF)
    cut = lambda c: wide[:, c:c + 128].unflatten(1, (2, 64))  # noqa: E731
    call = (lambda k, v, s: api.dlm_kv8_write(cpu_cache, k, v, off, start, s)) if write else (lambda k, v, s: api.dlm_kv8_read(cpu_cache, off, start, s, k=k, v=v))
    plain = all(type(x) in (list, tuple) and all(type(i) is int and i < 2**31 for i in x) for x in (off, start)) and len(off) > len(start) <= 32
    for slot in (None, [1, 0] * 20, torch.tensor([1, 0] * 20), [1]):
        for pair, ok in (((k, v), True), ((cut(0), cut(128)), True), ((k, cut(0)), False), ((k.float(), v), False), ((k.float(), v.float()), True), ((k.half(), v.half()), False),
                         ((k[:, :1], v[:, :1]), False), ((k[..., :32], v[..., :32]), False), ((k.transpose(1, 2).contiguous().transpose(1, 2), v), False),
                         ((k[:5], v), False), ((k[:1], v[:1]), True)):
            a, b = both(lambda: call(*pair, slot))
            assert a == b
            assert both.taken == (ok and plain and (slot is None or (type(slot) is list and len(slot) >= len(start))) and off[len(start)] <= len(pair[0]))
            if ok and plain and slot is None and len(pair[0]) == 6:
                assert (type(a) is list and len(a) == 1) == (off[len(start)] <= 6)
    both.status = -2
    assert both(lambda: api.dlm_kv8_write(cpu_cache, k, v, [0, 3], [0])) == [api.DlmError, api.DlmError] and both.taken


@pytest.mark.parametrize("off,keys", LISTS)
def test_attention_calls_either_way(both, cpu_cache, off, keys):
    q, out, mask = torch.zeros(6, 4, 64), torch.zeros(6, 4, 64), torch.zeros(6, 2, dtype=torch.int32)
    wide = torch.zeros(6, 300)[:, 4:260].unflatten(1, (4, 64))
    plain = all(type(x) in (list, tuple) and all(type(i) is int and i < 2**31 for i in x) for x in (off, keys)) and len(off) > len(keys) <= 32 and off[len(keys)] <= 6
    ws = torch.zeros(64, dtype=torch.uint8)
    for kw, ok in ((dict(q=q), True), (dict(q=wide), True), (dict(q=q, mask=mask), True), (dict(q=q, workspace=ws), True), (dict(q=q.to(BF)), False),
                   (dict(q=q.to(BF), out=out.to(BF)), True), (dict(q=q, out=wide), False), (dict(q=q, out=None), False), (dict(q=q, out=out[:5]), False),
                   (dict(q=q, mask=mask.long()), False), (dict(q=q, mask=mask[:4]), False), (dict(q=q, mask=mask.t()), False), (dict(q=q[..., :32]), False),
                   (dict(q=q[:, :, None]), False), (dict(q=q.to(torch.int32), out=out.to(torch.int32)), False)):
        kw = dict(dict(row_offsets=off, n_keys=keys, out=out), **kw)
        a, b = both(lambda: api.dlm_kv8_attention(cpu_cache, **kw))
        if kw["out"] is None and type(a) is list:  # (a new one each time)
            a, b = ([c[:3] + c[4:] for c in x] for x in (a, b))
        assert a == b and both.taken == (ok and plain)
    # a call that may need a workspace and has none is not the extension's
    both.status = -3
    seen = both(lambda: api.dlm_kv8_attention(cpu_cache, q, [0, 3], [5], out=out, workspace=ws))
    assert seen == [api.DlmError, api.DlmError] and both.taken


def test_norm_rope_calls_either_way(both):
    x, pos, g = torch.zeros(6, 400), torch.zeros(6, dtype=torch.int32), torch.ones(64)
    base = dict(x=x, positions=pos, n_q=2, n_kv=1, head_dim=64, q_gain=g, k_gain=g, eps=1e-5, theta=1e4, out=torch.zeros(6, 192))
    for change, ok in (({}, True), (dict(out=x), True), (dict(out=torch.zeros(6, 500)[:, :200]), True), (dict(x=x[:, 8:]), True), (dict(q_gain=None, k_gain=None), True),
                       (dict(out=torch.zeros(5, 192)), False), (dict(out=torch.zeros(6, 191)), False), (dict(out=torch.zeros(6, 192, dtype=BF)), False),
                       (dict(x=x[:, :191]), False), (dict(x=x.t()), False), (dict(positions=pos.long()), False), (dict(positions=pos[:5]), False),
                       (dict(positions=torch.zeros(12, dtype=torch.int32)[::2]), False), (dict(q_gain=torch.ones(32)), False), (dict(k_gain=g.to(BF)), False),
                       (dict(q_gain=torch.ones(128)[::2]), False), (dict(eps=1), False), (dict(theta=500000.0), True), (dict(x=x.half()), False)):
        a, b = both(lambda: api.dlm_qk_norm_rope(**dict(base, **change)))
        assert a == b and both.taken == ok, change
        assert (type(a) is list and len(a) == 1) == (ok or change == dict(eps=1)), change
