"""CPU checks of the compiled marshalling of placing, norm and adapters: every argument arrives where the C interface has it, and
what it does not take itself ends as the ctypes functions end it."""
import ctypes
import os

import pytest

import paper_2206_09557_amd as L
from paper_2206_09557_amd import lutgemm as M

pytestmark = pytest.mark.skipif("LUTGEMM_LIB" in os.environ, reason="a host-only build has no device calls")

BIG = (1 << 63) + 5      # an address beyond the signed range
WIDE = (1 << 40) + 1
P, I, I64, F, U, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_uint, ctypes.c_size_t
TYPES = {"lutgemm_kv_place": [P] * 3 + [I] * 2 + [P] * 5,
         "lutgemm_kv_trim": [P] * 3,
         "lutgemm_rms_norm": [P] * 6 + [I] * 3 + [I64] * 3 + [F, U, P],
         "lutgemm_adapt": [P] * 6 + [I] * 2 + [I64] * 3 + [U, P, S, P]}


class Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.fixture
def caught():
    """Calls of the entry points end in Python functions that keep their arguments and return code[0]."""
    calls, code = [], [0]
    assert set(TYPES) == set(M._STEP_CALLS)

    def catcher(name):
        def f(*args):
            calls.append((name, args))
            return code[0]
        return ctypes.CFUNCTYPE(ctypes.c_int, *TYPES[name])(f)

    L.lib()
    keep = {name: catcher(name) for name in TYPES}
    M._binding.load({name: ctypes.cast(f, ctypes.c_void_p).value for name, f in keep.items()})
    yield calls, code
    names = M._DEVICE_CALLS + M._CACHE_CALLS + M._STEP_CALLS
    M._binding.load({name: ctypes.cast(getattr(L.lib(), name), ctypes.c_void_p).value for name in names})


CASES = [("lutgemm_kv_place", (Buffer(16), 32, Buffer(BIG), 5, -6, 48, None, Buffer(64), 80), (16, 32, BIG, 5, -6, 48, None, 64, 80)),
         ("lutgemm_kv_trim", (Buffer(16), Buffer(BIG)), (16, BIG)),
         ("lutgemm_rms_norm", (Buffer(16), None, Buffer(BIG), 48, Buffer(64), None, 5, 6, 128, WIDE, -7, WIDE + 2, 0.125, 0xfffffffe),
          (16, None, BIG, 48, 64, None, 5, 6, 128, WIDE, -7, WIDE + 2, 0.125, 0xfffffffe)),
         ("lutgemm_adapt", (Buffer(16), 32, Buffer(BIG), 48, None, Buffer(80), 5, -6, WIDE, -7, WIDE + 2, 9, Buffer(96), 1 << 41),
          (16, 32, BIG, 48, None, 80, 5, -6, WIDE, -7, WIDE + 2, 9, 96, 1 << 41))]


@pytest.mark.parametrize("name,args,seen", CASES, ids=[c[0] for c in CASES])
def test_arguments_arrive(caught, name, args, seen):
    calls, code = caught
    f = getattr(L, name)
    assert f is getattr(M._binding, name)
    assert f(*args) is None and f(*args, 0) is None and f(*args, 4096) is None
    assert calls == [(name, seen + (s,)) for s in (None, None, 4096)]
    code[0] = L.LUTGEMM_EUNSUPPORTED
    with pytest.raises(L.LutGemmError) as e:
        f(*args)
    assert e.value.code == L.LUTGEMM_EUNSUPPORTED and name in str(e.value)


@pytest.mark.parametrize("name,args,seen", CASES, ids=[c[0] for c in CASES])
def test_what_is_left_to_ctypes(caught, name, args, seen):
    calls, _ = caught
    f = getattr(L, name)
    for wrong in ((), args[:-1], args + (0, 0), args[:-1] + ("text",), ("text",) + args[1:]):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            f(*wrong)
    assert calls == []


def test_each_set_is_loaded_without_the_others(caught):
    calls, _ = caught
    M._binding.load({})
    L.lutgemm_kv_trim(16, 32)
    assert calls == [("lutgemm_kv_trim", (16, 32, None))]


def test_by_name_through_ctypes():
    with pytest.raises(L.LutGemmError) as e:
        L.lutgemm_rms_norm(x=None, residual=None, weight=None, sum=None, y=None, scales=None, tokens=1, n=1, group=0, x_stride=1, stream_stride=1, y_stride=1,
                           eps=1, flags=0)
    assert e.value.code == L.LUTGEMM_EINVAL
