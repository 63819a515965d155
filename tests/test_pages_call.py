"""The CPython entries to the calls over caches in pages pass on what the tensors hold and refuse what the C functions cannot see, checked on the host against
stand-ins for the C functions."""
import ctypes as C
import re

import numpy as np
import pytest

from paper_2504_09261_amd import binding
from tests.test_ops_call import BF16, F32, I32, INFO, Rows, Tensor, addr, struct

SEEN = []
PAGES = [f for f, _ in binding.hack_pages._fields_]


class Shared(C.Structure):
    _fields_ = [("first", C.c_int32), ("count", C.c_int32), ("rows", C.c_int32)]


def pages_struct(p):
    return tuple(getattr(p[0], f) for f in PAGES)


PR, PP = C.POINTER(Rows), C.POINTER(binding.hack_pages)


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, PR, PR, PR, C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, PP, C.c_void_p)
def append_fn(*a):
    SEEN.append((*a[:3], struct(a[3]), struct(a[4]), struct(a[5]), *a[6:12], pages_struct(a[12]), a[13]))
    return -2


@C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, PP, C.c_void_p, C.c_int32, C.POINTER(Shared), C.c_int32, C.c_float, C.c_void_p,
             C.c_void_p)
def attn_fn(*a):
    SEEN.append((*a[:5], pages_struct(a[5]), *a[6:8], [(s.first, s.count, s.rows) for s in a[8][:a[9]]], *a[10:]))
    return 0


@pytest.fixture(autouse=True)
def entries():
    binding.load_library()
    SEEN.clear()


STRUCT = binding.hack_pages(1024, 2048, 9, 16, 3200, 192, 64, 512, 5, 6, 640, 0, 70)     # one, so that its address stays
FIELDS = (1024, 2048, 9, 16, 3200, 192, 64, 512, 5, 6, 640, 0, 70)


def info(device=1, dtype=BF16, head_dim=64, heads=3, rows=2):
    return (C.addressof(STRUCT), device, dtype, head_dim, heads, rows)


def append(q=None, q_out=None, qw=None, k=Tensor(16, (2, 3, 7, 64)), kw=None, v=Tensor(32, (2, 3, 7, 64)), norm=-1, eps=0.5, rope=99, axes=1, pos=None, fresh=None,
           cache=None):
    return binding._ops_call.append_pages(addr(append_fn), 2**47, INFO, q, q_out, qw, k, kw, v, norm, eps, rope, axes, pos, fresh, cache or info(), 77)


K, V = (16, None, 3, 1344, 448, 64, None, 0), (32, None, 3, 1344, 448, 64, None, 0)


def test_appending_arrives_as_given():
    assert append() == -2
    assert SEEN.pop() == (2**47, 2, 7, None, K, V, -1, 0.5, 99, None, 0, None, FIELDS, 77)
    q, out = Tensor(48, (2, 5, 7, 64), stride=(9999, 64, 320, 1)), Tensor(80, (2, 5, 7, 64))
    assert append(q, out, Tensor(96, (5, 64), F32), kw=Tensor(112, (64,), F32), norm=1, pos=Tensor(64, (2, 1, 7), I32), fresh=Tensor(8, (2,), I32)) == -2
    assert SEEN.pop() == (2**47, 2, 7, (48, 80, 5, 9999, 64, 320, 96, 64), K[:6] + (112, 0), V, 1, 0.5, 99, 64, 7, 8, FIELDS, 77)
    assert append(rope=None, pos=Tensor(64, (1,), F32)) == -2 and SEEN.pop()[8:11] == (None, None, 0)        # positions are not looked at without a rope
    # pages of one head: tables by head
    assert append(cache=info(heads=1, rows=6)) == -2 and SEEN.pop()[12] == FIELDS[:11] + (1, 70)
    assert STRUCT.by_head == 0


@pytest.mark.parametrize("kw", [
    dict(k=Tensor(16, (2, 3, 7, 64), F32)), dict(k=Tensor(16, (2, 3, 7, 128))), dict(v=Tensor(32, (2, 3, 6, 64))), dict(v=Tensor(32, (1, 3, 7, 64))), dict(v=Tensor(32, (2, 3, 7, 64), device=0)),
    dict(q=Tensor(48, (2, 5, 6, 64)), q_out=Tensor(80, (2, 5, 6, 64))), dict(q=Tensor(48, (2, 5, 7, 64)), q_out=Tensor(80, (2, 5, 8, 64))),
    dict(q=Tensor(48, (2, 5, 7, 64)), q_out=Tensor(80, (2, 5, 7, 64), stride=(2240, 64, 320, 1))), dict(kw=Tensor(96, (64,))), dict(pos=Tensor(64, (6,), I32)),
    dict(fresh=Tensor(8, (3,), I32)), dict(fresh=Tensor(8, (2,), F32)), dict(fresh=Tensor(8, (2, 1), I32)), dict(cache=info(device=0)), dict(cache=info(dtype=F32)),
    dict(cache=info(head_dim=128)), dict(cache=info(heads=2)), dict(cache=info(rows=3)), dict(cache=info(rows=6)), dict(cache=info(heads=1)), dict(cache=(1, 2, 3)), dict(cache=5),
])
def test_appending_that_is_refused(kw):
    with pytest.raises(AssertionError):
        append(**kw)
    assert not SEEN


def attn(q=Tensor(16, (2, 6, 7, 64)), out=None, cache=None, fresh=None, causal=False, shared=None, scale=0.25):
    return binding._ops_call.attn_pages(addr(attn_fn), 2**47, INFO, q, cache or info(), fresh, causal, shared, scale, out or Tensor(48, q.shape), 77)


def test_attention_arrives_as_given():
    assert attn() == 0
    assert SEEN.pop() == (2**47, 2, 7, 6, 16, FIELDS, None, 0, [], 0.25, 48, 77)
    assert attn(fresh=Tensor(8, (2,), I32), causal=True, shared=[(0, 1, 5), np.array([1, 1, 9])]) == 0
    assert SEEN.pop()[6:9] == (8, 1, [(0, 1, 5), (1, 1, 9)])
    assert attn(shared=()) == 0 and SEEN.pop()[8] == []
    assert attn(shared=tuple((i, 1, 1) for i in range(256))) == 0 and len(SEEN.pop()[8]) == 256


@pytest.mark.parametrize("kw", [
    dict(q=Tensor(16, (2, 4, 7, 64))), dict(q=Tensor(16, (6, 7, 64))), dict(q=Tensor(16, (2, 6, 7, 128))), dict(q=Tensor(16, (2, 6, 7, 64), F32)), dict(out=Tensor(48, (2, 6, 8, 64))),
    dict(q=Tensor(16, (2, 6, 7, 64), stride=(9, 9, 9, 1))), dict(q=Tensor(16, (1, 6, 7, 64))), dict(shared=[(0, 1)]), dict(shared=[(0, 1, 1)] * 257), dict(cache=info(rows=4)),
    dict(fresh=Tensor(8, (1,), I32)),
])
def test_attention_that_is_refused(kw):
    with pytest.raises(AssertionError):
        attn(**kw)
    assert not SEEN


def test_wrong_calls():
    with pytest.raises(TypeError, match=re.escape("takes 17 arguments")):
        binding._ops_call.append_pages(1, 2)
    with pytest.raises(TypeError, match=re.escape("takes 11 arguments")):
        binding._ops_call.attn_pages(1, 2)
    for bad in (5, [5], [(0, "x", 1)], [(0, 1.5, 1)]):
        with pytest.raises(TypeError):
            attn(shared=bad)
    for number in (2**31, -2**31 - 1, 2**64):
        with pytest.raises(OverflowError):
            attn(shared=[(0, 1, number)])
    with pytest.raises(TypeError):
        attn(scale="x")
    assert not SEEN


def test_groups_that_change_while_they_are_read():
    groups = []

    class Clears:
        def __init__(self, n, what):
            self.n, self.what = n, what

        def __index__(self):
            self.what.clear()
            return self.n
    inner = []
    inner += [Clears(0, inner), 1, 5]
    groups += [inner, (Clears(1, groups), 1, 9), (2, 1, 3)]
    assert attn(shared=groups) == 0
    assert SEEN.pop()[8] == [(0, 1, 5), (1, 1, 9), (2, 1, 3)] and not groups and not inner
