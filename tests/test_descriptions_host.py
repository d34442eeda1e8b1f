"""CPU-only checks of the binding's descriptions of tensors: what they hold is freed with them."""
import gc
import weakref

import pytest
import torch


@pytest.fixture(scope="module")
def E():
    from paper_2502_06833_b200 import build
    build.build()
    from paper_2502_06833_b200 import binding
    return binding


def _matrix(E):
    return E.ead_e4m3_matrix(torch.zeros(3, 160, dtype=torch.uint8), torch.zeros(3, 5, dtype=torch.uint8), block=(1, 32))


def _rope(E):
    return E.ead_rope(torch.zeros(32), 64, q_weight=torch.zeros(64, dtype=torch.bfloat16))


def _cache(E):
    k, v = (torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16) for _ in "kv")
    return E.ead_kv_cache(k, v)


def _batch(E):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)                  # noqa: E731
    return E.ead_kv_batch(torch.zeros(1, 4, dtype=torch.int32), i32(0, 2), i32(9), n_tokens=2, max_new=2, max_len=9)


@pytest.mark.parametrize("make", [_matrix, _rope, _cache, _batch])
def test_tensors_go_with_their_description(E, make):
    """Without the cyclic collector, which counts Python objects and knows nothing of the memory of a device behind them."""
    gc.collect()
    on = gc.isenabled()
    gc.disable()
    try:
        d = make(E)
        held = [weakref.ref(t) for t in d.held if t is not None]
        assert held and all(r() is not None for r in held)              # borrowed: the description alone keeps them
        del d
        assert not any(r() is not None for r in held)
    finally:
        if on:
            gc.enable()


@pytest.mark.parametrize("make", [_matrix, _rope, _cache, _batch])
def test_what_is_passed_on_is_the_description(E, make):
    """Fields that change later are what a call sees."""
    import ctypes as C
    d = make(E)
    name = type(d)._fields_[0][0]
    setattr(d, name, 12345)
    assert getattr(C.cast(d.ref, C.POINTER(type(d))).contents, name) == 12345
