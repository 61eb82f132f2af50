"""CPU checks of the compiled marshalling of rotary positions, cache and attention: every argument arrives where the C
interface has it, and what it does not take itself ends as the ctypes functions end it."""
import ctypes
import os

import pytest

import paper_2206_09557_amd as L
from paper_2206_09557_amd import lutgemm as M

pytestmark = pytest.mark.skipif("LUTGEMM_LIB" in os.environ, reason="a host-only build has no device calls")

BIG = (1 << 63) + 5      # an address beyond the signed range
P, I, I64, F, U, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_uint, ctypes.c_size_t
TYPES = {"lutgemm_rope": [P] * 4 + [I] * 4 + [I64] * 2 + [F, U, P],
         "lutgemm_kv_write": [P] * 5 + [I64] * 2 + [P],
         "lutgemm_kv_read": [P] * 4 + [I64] * 2 + [P],
         "lutgemm_attention": [P] * 5 + [I, I64, I64, F, I64, P, S, P]}
WIDE = (1 << 40) + 1


class Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.fixture
def caught():
    """Calls of the entry points end in Python functions that keep their arguments and return code[0]."""
    calls, code = [], [0]
    assert set(TYPES) == set(M._CACHE_CALLS)

    def catcher(name):
        def f(*args):
            calls.append((name, args))
            return code[0]
        return ctypes.CFUNCTYPE(ctypes.c_int, *TYPES[name])(f)

    L.lib()
    keep = {name: catcher(name) for name in TYPES}
    M._binding.load({name: ctypes.cast(f, ctypes.c_void_p).value for name, f in keep.items()})
    yield calls, code
    names = M._DEVICE_CALLS + M._CACHE_CALLS
    M._binding.load({name: ctypes.cast(getattr(L.lib(), name), ctypes.c_void_p).value for name in names})


CASES = [("lutgemm_rope", (Buffer(16), 32, Buffer(BIG), 48, 5, 6, 128, 64, WIDE, -7, 0.5, 0xfffffffe),
          (16, 32, BIG, 48, 5, 6, 128, 64, WIDE, -7, 0.5, 0xfffffffe)),
         ("lutgemm_kv_write", (Buffer(16), None, Buffer(BIG), 48, Buffer(64), WIDE, -7), (16, None, BIG, 48, 64, WIDE, -7)),
         ("lutgemm_kv_read", (Buffer(16), 32, None, Buffer(BIG), WIDE, -7), (16, 32, None, BIG, WIDE, -7)),
         ("lutgemm_attention", (Buffer(16), None, Buffer(BIG), 48, 64, 7, WIDE, -7, -0.125, WIDE + 1, Buffer(80), 1 << 41),
          (16, None, BIG, 48, 64, 7, WIDE, -7, -0.125, WIDE + 1, 80, 1 << 41))]


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
    """Nothing reaches the library, or ctypes calls it (the real one: which refuses these addresses' null companions)."""
    calls, _ = caught
    f = getattr(L, name)
    for wrong in ((), args[:-1], args + (0, 0), args[:-1] + ("text",), ("text",) + args[1:]):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            f(*wrong)
    assert calls == []


def test_a_whole_number_as_the_scale(caught):
    """ctypes takes an int for a float; the call is its own then, and the library's refusal is raised."""
    calls, _ = caught
    with pytest.raises(L.LutGemmError) as e:
        L.lutgemm_attention(None, None, None, None, None, 1, 128, 128, 1, 0, None, 0)
    assert e.value.code == L.LUTGEMM_EINVAL and calls == []


def test_either_set_is_loaded_without_the_other(caught):
    calls, _ = caught
    M._binding.load({})
    L.lutgemm_kv_read(16, 32, None, 48, 1, 2)
    assert calls == [("lutgemm_kv_read", (16, 32, None, 48, 1, 2, None))]
