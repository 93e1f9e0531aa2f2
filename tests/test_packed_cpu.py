"""Packed caches without a GPU: the memory model, the refusals that come before any CUDA call, the format itself."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2412_05693_b200 as bm
from paper_2412_05693_b200.build import build
from tests import packed_reference as ref


@pytest.fixture(scope="module", autouse=True)
def built():
    build()


def cfg(**kw):
    base = dict(batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128, capacity=1024)
    base.update(kw)
    return bm.PackedConfig(**base)


def test_memory_model():
    assert bm.packed_bytes_per_sample(cfg()) == 8 * 1024 * 2 * 72
    assert bm.packed_bytes_per_sample(cfg(capacity=1025, n_layers=3, head_dim=64, dtype="f32")) == 3 * 8 * 1056 * 2 * 36
    assert bm.packed_arena_bytes(cfg()) == 256 + 16 * 8 * 1024 * 144
    for budget in (100, 3 << 30, 40 << 30):
        b = bm.packed_max_batch(cfg(), budget)
        assert (b == 0 or bm.packed_arena_bytes(cfg(batch=b)) <= budget) and bm.packed_arena_bytes(cfg(batch=b + 1)) > budget
    # the same rows in bf16 take 3.6 times as much
    plain = bm.Config(batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128, kv_max=1023, block_max=512)
    assert bm.cache_bytes_per_sample(plain) / bm.packed_bytes_per_sample(cfg()) == pytest.approx(520 / 144)
    assert bm.packed_workspace_bytes(cfg()) <= bm.packed_workspace_bytes(cfg(queries_max=64))


@pytest.mark.parametrize("bad", [dict(n_kv_heads=5), dict(head_dim=96), dict(capacity=0), dict(capacity=(1 << 24) + 1), dict(queries_max=0),
                                 dict(n_layers=0), dict(n_kv_heads=0), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
                                 dict(softmax_scale=float("inf")), dict(device=-1), dict(batch=0)])
def test_invalid_configs_are_rejected(bad):
    for query in (bm.packed_arena_bytes, bm.packed_workspace_bytes):
        with pytest.raises(bm.BMError) as e:
            query(cfg(**bad))
        assert e.value.code == 1


def test_sizes_beyond_a_size_t_are_rejected():
    huge = cfg(batch=2 ** 31 - 1, n_layers=2 ** 31 - 1, n_kv_heads=2 ** 20, n_q_heads=2 ** 20, capacity=1 << 24)
    with pytest.raises(bm.BMError):
        bm.packed_arena_bytes(huge)


def test_null_and_misaligned_arguments_are_refused_before_any_cuda_call():
    L, h, c = bm.lib(), C.c_void_p(None), cfg().c()
    need = bm.packed_arena_bytes(cfg())
    assert L.bm_packed_create(C.byref(c), None, need, None, C.byref(h)) == 1
    assert L.bm_packed_create(C.byref(c), C.c_void_p(0x1010), need, None, C.byref(h)) == 1
    assert L.bm_packed_create(C.byref(c), C.c_void_p(0x1000), need - 1, None, C.byref(h)) == 2
    assert L.bm_packed_create(C.byref(c), C.c_void_p(0x1000), need, None, None) == 1
    assert L.bm_packed_destroy(None) == 1
    assert L.bm_packed_write(None, 0, 0, 1, C.c_void_p(16), C.c_void_p(16), None, 1, None, None, None) == 1
    assert L.bm_packed_write_from(None, 0, 0, 1, None, 0, 0, None) == 1
    assert L.bm_packed_read(None, 0, 0, 1, 0, 1, None, C.c_void_p(16), C.c_void_p(16), None) == 1
    assert L.bm_packed_attend(None, 0, 0, 1, C.c_void_p(16), None, 1, C.c_void_p(16), None, 0, C.c_void_p(16), C.c_void_p(16), 1 << 30,
                              None) == 1
    w = C.c_int32(0)
    assert L.bm_packed_status(None, C.byref(w), None) == 1 and L.bm_packed_clear_status(None, None) == 1


def test_the_format_itself():
    """Hand-worked groups, and the step of an eighth of the peak as the largest error of what is not clamped."""
    x = np.zeros((1, 64))
    x[0, :4] = [-8.0, 7.0, 0.5, 1.5]
    x[0, 32:35] = [4.0, -4.0, 3.9]
    code, s = ref.quantise(x)
    assert s.tolist() == [[1.0, -0.5]]
    assert code[0, 0, :4].tolist() == [-8, 7, 0, 2] and code[0, 1, :3].tolist() == [-8, 7, -8]
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(500, 128, generator=gen, dtype=torch.float64)
    code, s = ref.quantise(x)
    err = np.abs(ref.values(code, s).numpy() - x.numpy()).reshape(500, 4, 32)
    assert (err[np.abs(code) < 7] <= np.broadcast_to(np.abs(s)[..., None], err.shape)[np.abs(code) < 7] * 0.5000001).all()
    # fp32 tells a quotient apart from a tie: no quotient of 24 by 11 bits rounds to one that it is not
    s = (torch.randint(1024, 2048, (20000,), generator=gen).double()) / 1024
    k = torch.randint(0, 8, (20000,), generator=gen).double() + 0.5
    t = (k * s).float()
    assert torch.equal(t.double(), k * s)
    for x in (torch.nextafter(t, torch.full_like(t, 100.0)), torch.nextafter(t, torch.zeros_like(t))):
        assert ((x / s.float()).double() != k).all()
