"""What the 4-bit and window calls refuse before they reach a GPU: the library without a context, and the binding with
arguments of the wrong type, place or size."""
import ctypes
import os
import re

import pytest
import torch

from paper_2609_04971_gb300 import _build, bkv

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bkv.h")
CALLS = ("bkv_pack4", "bkv_unpack4", "bkv_attend4", "bkv_attend4_reserve", "bkv_evict4", "bkv_attend_window")


def test_declared_exported_and_bound():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    bkv.load_library()
    raw = ctypes.CDLL(_build.LIB_PATH)
    for name in CALLS:
        assert re.search(rf"\b{name}\s*\(", src) and hasattr(raw, name) and hasattr(bkv, name)


def test_without_a_context():
    lib = bkv.load_library()
    for name in CALLS:
        fn = getattr(lib, name)
        args = [None] + [0.0 if t is ctypes.c_double else None if t is ctypes.c_void_p else 1 for t in fn.argtypes[1:]]
        assert fn(*args) == bkv.BKV_EINVAL, name


@pytest.fixture
def bk():
    """A binding object of batch 2, 4 query heads, 2 KV heads of 64 and capacity 10, without a context behind it."""
    o = bkv.BeaconKV.__new__(bkv.BeaconKV)
    o.cfg = bkv.BkvConfig(1, 2, 4, 2, 64, 1, 0, 0, 10, 0.0, 0)
    o.ctx, o.n_inst, o._layer = None, 4, (2, 4, 64, 4, 40)
    bkv.load_library()
    return o


def test_binding_refuses_what_is_not_on_the_gpu(bk):
    q, K = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 10, 64, dtype=torch.bfloat16)
    K4, S4 = torch.zeros(2, 2, 10, 32, dtype=torch.uint8), torch.zeros(2, 2, 10, 2, 2, 2, dtype=torch.float16)
    n = torch.zeros(2, 2, dtype=torch.int32)
    for call in (lambda: bk.attend4(q, K4, K4, S4, length=n), lambda: bk.attend_window(q, K, K, length=n, window=3),
                 lambda: bk.pack4(K, K, K4, K4, S4, length=n), lambda: bk.unpack4(K4, K4, S4, K, K, length=n),
                 lambda: bk.evict4(K4, K4, S4, torch.zeros(2, 2, 10), L=n, budget=5)):
        with pytest.raises(TypeError):
            call()


def test_binding_refuses_wrong_sizes(bk):
    bad = torch.zeros(7)
    q, K = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 10, 64, dtype=torch.bfloat16)
    for call in (lambda: bk.attend4(q, bad, bad, bad, length=bad),
                 lambda: bk.attend_window(q, bad, K, length=bad, window=3),
                 lambda: bk.pack4(K[:1], K, bad, bad, bad, length=bad),
                 lambda: bk.pack4(K[0], K, bad, bad, bad, length=bad),
                 lambda: bk.unpack4(bad, bad, bad, K[:, :1], K, length=bad),
                 lambda: bk.evict4(bad, bad, bad, bad, L=bad, budget=5, K4_out=bad),
                 lambda: bk.evict4(bad, bad, bad, bad, L=bad, budget=5)):
        with pytest.raises(ValueError):
            call()
