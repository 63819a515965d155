"""The CPython entries to the operators around the cache pass on what the tensors hold and refuse what the C functions cannot see, checked on the host
against stand-ins for the C functions."""
import ctypes as C
import re

import numpy as np
import pytest

from paper_2504_09261_amd import binding

BF16, F32, I32, U8 = "bf16", "f32", "i32", "u8"     # compared by identity only
INFO = (64, 3, 1, BF16, F32, I32, U8)               # head_dim, heads, device, element types


class Tensor:
    def __init__(self, ptr, shape, dtype=BF16, device=1, stride=None):
        self.ptr, self.shape, self.dtype, self.device = ptr, tuple(shape), dtype, device
        dense = tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))
        self.strides, self.dense = stride or dense, stride in (None, dense)

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.dense

    def stride(self):
        return self.strides

    def data_ptr(self):
        return self.ptr


class Rows(C.Structure):
    _fields_ = [("x", C.c_void_p), ("out", C.c_void_p), ("heads", C.c_int32), ("stride_b", C.c_int64), ("stride_h", C.c_int64),
                ("stride_n", C.c_int64), ("weight", C.c_void_p), ("weight_stride_h", C.c_int64)]


def struct(p):
    return None if not p else tuple(getattr(p[0], f) for f, _ in p[0]._fields_)


def cache_struct(p, n):
    return None if not p else (p[0].k, p[0].v, C.cast(p[0].pos, C.c_void_p).value, p[0].rows, p[0].off[:n], p[0].len[:n])


SEEN = []
PC = C.POINTER(binding.hack_cache)


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(Rows), C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p)
def rotate_fn(*a):
    SEEN.append((*a[:3], struct(a[3]), *a[4:]))
    return -4


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(Rows), C.POINTER(Rows), C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32,
             C.c_void_p)
def norm_fn(*a):
    SEEN.append((*a[:3], struct(a[3]), struct(a[4]), *a[5:]))
    return -3


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, PC, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.POINTER(C.c_int32), PC, C.c_void_p)
def pack_fn(*a):
    SEEN.append((*a[:3], cache_struct(a[3], 6), *a[4:9], a[9][:6] if a[9] else None, cache_struct(a[10], 6), a[11]))
    return 0


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, PC, C.POINTER(C.c_int32), PC, C.c_void_p)
def unpack_fn(*a):
    SEEN.append((*a[:2], cache_struct(a[2], 6), a[3][:6] if a[3] else None, cache_struct(a[4], 6), a[5]))
    return 0


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, PC, C.c_float, C.c_void_p, C.c_void_p)
def attn_fn(*a):
    SEEN.append((*a[:4], cache_struct(a[4], 6), *a[5:]))
    return 0


def addr(f):
    return C.cast(f, C.c_void_p).value


@pytest.fixture(autouse=True)
def entries():
    binding.load_library()
    SEEN.clear()
    return binding._ops_call


def rotate(x=Tensor(16, (2, 5, 7, 64)), out=Tensor(32, (2, 5, 7, 64)), w=None, k=None, k_out=None, kw=None, norm=-1, eps=0.0, rope=99, axes=1, pos=None, pos0=3):
    return binding._ops_call.rotate(addr(rotate_fn if norm < 0 else norm_fn), 2**47, INFO, x, out, w, k, k_out, kw, norm, eps, rope, axes, pos, pos0, 77)


def test_rotations_arrive_as_given():
    assert rotate() == -4
    assert SEEN.pop() == (2**47, 2, 7, (16, 32, 5, 5 * 7 * 64, 7 * 64, 64, None, 0), 99, None, 0, 3, 77)
    x = Tensor(16, (1, 5, 1, 64), stride=(-1, 64, 12345, 1))       # dimensions of one element: any stride
    assert rotate(x, Tensor(32, (1, 5, 1, 64)), pos=Tensor(64, (1,), I32)) == -4
    assert SEEN.pop()[3:7] == ((16, 32, 5, 0, 64, 0, None, 0), 99, 64, 0)
    x = Tensor(16, (2, 5, 7, 64), stride=(9999, 64, 640, 1))
    for axes, shape, stride in ((1, (7,), 0), (1, (1, 7), 0), (1, (2, 1, 7), 7), (2, (2, 7), 0), (2, (2, 2, 7), 14)):
        assert rotate(x, pos=Tensor(64, shape, I32), axes=axes) == -4
        got = SEEN.pop()
        assert got[3][3:6] == (9999, 64, 640) and got[5:7] == (64, stride)
    k, ko = Tensor(48, (2, 1, 7, 64)), Tensor(80, (2, 1, 7, 64))
    assert rotate(norm=1, eps=0.5, k=k, k_out=ko, w=Tensor(96, (5, 64), F32), kw=Tensor(112, (64,), F32)) == -3
    assert SEEN.pop() == (2**47, 2, 7, (16, 32, 5, 2240, 448, 64, 96, 64), (48, 80, 1, 448, 0, 64, 112, 0), 1, 0.5, 99, None, 0, 3, 77)
    assert rotate(norm=0, eps=1.0, rope=None, pos=Tensor(64, (3,), U8)) == -3     # positions are not looked at without a rope
    assert SEEN.pop()[4:10] == (None, 0, 1.0, None, None, 0)


@pytest.mark.parametrize("kw", [
    dict(x=Tensor(16, (2, 5, 7, 64), F32)), dict(x=Tensor(16, (2, 5, 7, 64), device=0)), dict(x=Tensor(16, (2, 5, 7, 64), device=-1)), dict(x=Tensor(16, (5, 7, 64))),
    dict(x=Tensor(16, (2, 5, 7, 128))), dict(x=Tensor(16, (2, 5, 7, 64), stride=(2240, 448, 1, 7))), dict(out=Tensor(32, (2, 5, 8, 64))), dict(out=Tensor(32, (2, 5, 7, 64), F32)),
    dict(out=Tensor(32, (2, 5, 7, 64), stride=(2240, 64, 320, 1))), dict(norm=0, w=Tensor(96, (64,))), dict(norm=0, w=Tensor(96, (4, 64), F32)), dict(norm=0, w=Tensor(96, (32,), F32)),
    dict(norm=0, k=Tensor(48, (2, 1, 6, 64)), k_out=Tensor(80, (2, 1, 6, 64))), dict(pos=Tensor(64, (6,), I32)), dict(pos=Tensor(64, (7,), F32)), dict(pos=Tensor(64, (7,), I32), axes=2),
    dict(pos=Tensor(64, (2, 7), I32)), dict(pos=Tensor(64, (2, 7, 1), I32, stride=(1, 2, 14))),
])
def test_rotations_that_are_refused(kw):
    with pytest.raises(AssertionError):
        rotate(**kw)
    assert not SEEN


def cache(rows=40, n=6, packed=False, pos=False, **kw):
    c = object.__new__(binding.PackedCache if packed else binding.Cache)
    width, dtype = (34 * 64, U8) if packed else (64, BF16)
    c.k, c.v = Tensor(1024, (rows, width), dtype), Tensor(2048, (rows, width), dtype)
    c.pos = Tensor(4096, (rows * (64 if packed else 1),), I32) if pos else None
    c.off, c.len = np.arange(n, dtype=np.int64) * 64, np.arange(n, dtype=np.int32)
    for name, v in kw.items():
        setattr(c, name, v)
    return c


OFF, LEN = [0, 64, 128, 192, 256, 320], [0, 1, 2, 3, 4, 5]


def pack(cache_in=None, k=Tensor(16, (2, 3, 4, 64)), v=Tensor(32, (2, 3, 4, 64)), kept=None, first=None, out=None, B=2, N=4):
    return binding._ops_call.pack(addr(pack_fn), 2**47, INFO, B, N, cache_in, k, v, 5, kept, first, out or cache(packed=True), 77)


def test_packed_calls_arrive_as_given():
    assert pack() == 0
    assert SEEN.pop() == (2**47, 2, 4, None, 16, 32, 5, None, 0, None, (1024, 2048, None, 2560, OFF, LEN), 77)
    assert pack(cache(pos=True), None, None, Tensor(8, (6, 33), I32), np.arange(6, dtype=np.int32), cache(packed=True, pos=True)) == 0
    assert SEEN.pop() == (2**47, 2, 4, (1024, 2048, 4096, 40, OFF, LEN), None, None, 5, 8, 33, LEN, (1024, 2048, 4096, 2560, OFF, LEN), 77)
    assert pack(first=np.arange(6)) == 0 and SEEN.pop()[9] == LEN                                     # int64 arrays as well
    assert pack(first=list(range(6))) is None and pack(first=np.arange(6.0)) is None and pack(first=np.arange(12)[::2]) is None and not SEEN     # the caller converts them
    un = lambda **kw: binding._ops_call.unpack(addr(unpack_fn), 2**47, INFO, 2, kw.get("packed") or cache(packed=True), kw.get("first"), kw.get("out") or cache(), 77)  # noqa: E731
    assert un(first=np.arange(6, dtype=np.int32)) == 0
    assert SEEN.pop() == (2**47, 2, (1024, 2048, None, 2560, OFF, LEN), LEN, (1024, 2048, None, 40, OFF, LEN), 77)
    assert un(first=np.arange(6)) == 0 and SEEN.pop()[3] == LEN
    assert un(first=list(range(6))) is None and not SEEN
    at = lambda q, kv=None: binding._ops_call.attn(addr(attn_fn), 2**47, INFO, q, kv or cache(packed=True), 0.25, Tensor(48, q.shape), 77)  # noqa: E731
    assert at(Tensor(16, (2, 12, 5, 64))) == 0
    assert SEEN.pop() == (2**47, 2, 20, 16, (1024, 2048, None, 2560, OFF, LEN), 0.25, 48, 77)
    for bad in (dict(packed=cache()), dict(out=cache(packed=True)), dict(first=np.arange(5, dtype=np.int32)), dict(out=cache(n=5)), dict(packed=cache(packed=True, n=7))):
        with pytest.raises(AssertionError):
            un(**bad)
    for q, kv in ((Tensor(16, (2, 4, 5, 64)), None), (Tensor(16, (2, 3, 5, 128)), None), (Tensor(16, (1, 3, 5, 64)), None), (Tensor(16, (2, 3, 5, 64), F32), None),
                  (Tensor(16, (2, 3, 5, 64)), cache())):
        with pytest.raises(AssertionError):
            at(q, kv)
    with pytest.raises(AssertionError):
        binding._ops_call.attn(addr(attn_fn), 2**47, INFO, Tensor(16, (2, 3, 5, 64)), cache(packed=True), 0.25, Tensor(48, (2, 3, 6, 64)), 77)
    assert not SEEN


@pytest.mark.parametrize("kw", [
    dict(k=Tensor(16, (2, 3, 5, 64))), dict(v=Tensor(32, (2, 3, 4, 64), F32)), dict(k=Tensor(16, (2, 3, 4, 64), device=0)), dict(B=1), dict(N=5), dict(kept=Tensor(8, (5, 33), I32)),
    dict(kept=Tensor(8, (6, 33), F32)), dict(kept=Tensor(8, (198,), I32)), dict(first=np.arange(5, dtype=np.int32)), dict(cache_in=cache(n=5)), dict(cache_in=cache(packed=True)),
    dict(cache_in=cache(k=Tensor(1024, (40, 128)))), dict(cache_in=cache(v=Tensor(2048, (41, 64)))), dict(cache_in=cache(off=np.arange(6, dtype=np.int32))),
    dict(cache_in=cache(len=np.arange(6))), dict(cache_in=cache(len=[0] * 6)), dict(out=cache(packed=True, pos=True, rows=30, k=Tensor(1024, (40, 34 * 64), U8), v=Tensor(2048, (40, 34 * 64), U8))),
    dict(out=cache(packed=True, off=np.arange(7, dtype=np.int64))),
])
def test_packs_that_are_refused(kw):
    with pytest.raises(AssertionError):
        pack(**kw)
    assert not SEEN


def test_wrong_calls():
    with pytest.raises(TypeError, match=re.escape("takes 16 arguments")):
        binding._ops_call.rotate(1, 2)
    with pytest.raises(AttributeError):
        rotate(x=5)
    with pytest.raises(TypeError):
        rotate(eps="x")
    with pytest.raises(AttributeError):
        pack(cache_in=7)


@pytest.mark.parametrize("number", [2**31, -2**31 - 1, 2**64])
def test_numbers_of_more_than_32_bits_are_refused(number):
    assert rotate(pos0=-2**31) == -4 and rotate(pos0=2**31 - 1) == -4
    assert [x[7] for x in SEEN] == [-2**31, 2**31 - 1]
    SEEN.clear()
    for f in (lambda: rotate(pos0=number), lambda: pack(N=number), lambda: pack(B=number)) + ((lambda: pack(first=np.full(6, number)),) if number < 2**63 else ()):
        with pytest.raises(OverflowError):
            f()
    assert not SEEN


def test_a_kept_list_of_no_columns_is_still_one():
    """torch gives tensors without elements the address 0, which the C function takes for no list: all rows in order."""
    assert pack(kept=Tensor(0, (6, 0), I32)) == 0
    call = SEEN.pop()
    assert call[7] and call[7] % 4 == 0 and call[8] == 0
    with pytest.raises(AssertionError):
        pack(kept=Tensor(0, (5, 0), I32))
    assert not SEEN


@pytest.mark.parametrize("rows", [np.full(12, 2**32 + 5)[::2], [2**32 + 5] * 6, np.full(6, 2.0**32 + 5), np.full(6, 5.5), np.full(6, np.nan), np.full(6, 2**31, np.uint32),
                                  [2**70] * 6, np.full(6, 2**64 - 1, np.uint64)],
                         ids=["strided", "list", "far float", "half", "nan", "uint32", "far list", "uint64"])
def test_row_numbers_that_32_bits_do_not_hold_are_refused(monkeypatch, rows):
    """Those that the entries leave to the caller, and lengths of a packed cache."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(binding, "_stream", lambda: 77)
    hk = object.__new__(binding.Hack)
    hk.ctx, hk._info, hk.lib = C.c_void_p(2**47), INFO, None
    monkeypatch.setitem(binding._ops_addr, "pack", addr(pack_fn))
    monkeypatch.setitem(binding._ops_addr, "unpack", addr(unpack_fn))
    new = dict(k_new=Tensor(16, (2, 3, 4, 64)), v_new=Tensor(32, (2, 3, 4, 64)))
    mem = torch.zeros((100, 34 * 64), dtype=torch.uint8)
    with pytest.raises(OverflowError):
        hk.pack(2, 4, cache(packed=True), at=rows, **new)
    with pytest.raises(OverflowError):
        hk.unpack(2, cache(packed=True), cache(), first=rows)
    with pytest.raises(OverflowError):
        binding.PackedCache(mem, mem, np.zeros(6), rows)
    assert not SEEN
    hk.pack(2, 4, cache(packed=True), at=np.arange(12)[::2], **new)
    hk.pack(2, 4, cache(packed=True), at=[0, 2, 4, 6, 8, 10], **new)
    hk.unpack(2, cache(packed=True), cache(), first=torch.arange(0, 12, 2))
    assert [c[9] for c in SEEN[:2]] == [[0, 2, 4, 6, 8, 10]] * 2 and SEEN[2][3] == [0, 2, 4, 6, 8, 10]
    assert list(binding.PackedCache(mem, mem, [0, 64], np.array([3.0, 4.0])).len) == [3, 4]
    for off in ([0.5, 64.0], np.array([2**64 - 64, 64], np.uint64)):
        with pytest.raises(OverflowError):
            binding.PackedCache(mem, mem, off, [1, 2])


def _freq_address(rope):
    s = C.cast(rope.address, C.POINTER(binding.hack_rope)).contents
    return C.cast(s.freq, C.c_void_p).value


def test_a_rope_keeps_what_its_structure_points_to():
    """The library reads frequencies, sizes and axes from the structure: they stay what the checks have seen, and alive, whatever becomes of the parts."""
    import copy
    import pickle
    freq = np.linspace(0.5, 2, 16)
    rope = binding.Rope(freq, 32, axes=2, layout="interleaved", gain=1.5)
    for r in (rope, copy.copy(rope), copy.deepcopy(rope), pickle.loads(pickle.dumps(rope))):
        s = C.cast(r.address, C.POINTER(binding.hack_rope)).contents
        assert (s.layout, s.rot_dim, s.axes, s.gain) == (1, 32, 2, 1.5) == (binding.ROPE_LAYOUTS[r.layout], r.rot_dim, r.axes, r.gain)
        assert s.freq[:16] == list(np.linspace(0.5, 2, 16)) == list(r.freq)
        assert _freq_address(r) == r.freq.ctypes.data
        assert r is rope or (r.address != rope.address and _freq_address(r) != _freq_address(rope))
    for name, value in (("freq", np.zeros(16)), ("axes", 1), ("rot_dim", 16), ("layout", "half"), ("gain", 1.0), ("address", 0)):
        with pytest.raises(AttributeError):
            setattr(rope, name, value)
    rope.freq[3] = 7.0     # in place: the structure points there
    assert C.cast(rope.address, C.POINTER(binding.hack_rope)).contents.freq[3] == 7.0
