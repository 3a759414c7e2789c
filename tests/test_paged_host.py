"""The paged cache's and the rotary table's argument checks, without a GPU: documented codes before any device work."""
import ctypes as C

import pytest

from paper_2504_10724_amd import capi as ee

DUMMY = C.c_void_p(4096)


def _rope(**kw):
    c = dict(head_dim=128, rot_dim=128, pairing=ee.EE_ROPE_HALF, max_pos=64, scaling=ee.EE_ROPE_UNSCALED, trained_pos=0, theta=10000.0,
             factor=1.0, low=1.0, high=4.0, magnitude=0.0)
    c.update(kw)
    return ee.ee_rope_config(**c)


@pytest.mark.parametrize("kw,code", [
    (dict(rot_dim=127), ee.EE_ERR_SHAPE), (dict(rot_dim=130), ee.EE_ERR_SHAPE), (dict(rot_dim=0), ee.EE_ERR_SHAPE),
    (dict(max_pos=0), ee.EE_ERR_SHAPE), (dict(pairing=2), ee.EE_ERR_INVALID_ARG), (dict(scaling=9), ee.EE_ERR_INVALID_ARG),
    (dict(theta=1.0), ee.EE_ERR_INVALID_ARG), (dict(theta=float("nan")), ee.EE_ERR_INVALID_ARG), (dict(theta=float("inf")), ee.EE_ERR_INVALID_ARG),
    (dict(scaling=ee.EE_ROPE_LINEAR, factor=0.0), ee.EE_ERR_INVALID_ARG), (dict(scaling=ee.EE_ROPE_BASE, rot_dim=2), ee.EE_ERR_SHAPE),
    (dict(scaling=ee.EE_ROPE_BANDS, factor=8.0), ee.EE_ERR_INVALID_ARG),
    (dict(scaling=ee.EE_ROPE_BANDS, factor=8.0, trained_pos=9, low=4.0), ee.EE_ERR_INVALID_ARG),
    (dict(magnitude=-1.0), ee.EE_ERR_INVALID_ARG), (dict(magnitude=float("nan")), ee.EE_ERR_INVALID_ARG),
])
def test_rope_configurations(kw, code):
    lib, h = ee.load(), C.c_void_p()
    assert lib.ee_rope_create(C.byref(_rope(**kw)), C.byref(h)) == code
    assert lib.ee_last_error() and not h.value


def _paged(**kw):
    c = dict(n_layers=2, n_pages=10, n_kv_heads=2, head_dim=128, page_size=64, dtype=ee.EE_BF16)
    c.update(kw)
    return ee.ee_paged_config(**c)


@pytest.mark.parametrize("kw,code", [
    (dict(n_layers=0), ee.EE_ERR_SHAPE), (dict(n_pages=0), ee.EE_ERR_SHAPE), (dict(n_kv_heads=0), ee.EE_ERR_SHAPE),
    (dict(page_size=16), ee.EE_ERR_SHAPE), (dict(page_size=48), ee.EE_ERR_SHAPE), (dict(page_size=8192), ee.EE_ERR_SHAPE),
    (dict(head_dim=100), ee.EE_ERR_SHAPE), (dict(head_dim=288), ee.EE_ERR_SHAPE), (dict(dtype=5), ee.EE_ERR_DTYPE),
    (dict(dtype=ee.EE_F32, head_dim=6), ee.EE_ERR_SHAPE), (dict(dtype=ee.EE_F32, head_dim=260), ee.EE_ERR_SHAPE),
    (dict(n_layers=2 ** 31 - 1, n_pages=2 ** 31 - 1, n_kv_heads=65535), ee.EE_ERR_SHAPE),
    (dict(n_layers=1, n_pages=2 ** 31 - 1, n_kv_heads=2, page_size=64), ee.EE_ERR_SHAPE),          # groups beyond 32 bits
])
def test_paged_configurations(kw, code):
    lib, h = ee.load(), C.c_void_p()
    assert lib.ee_paged_pool_bytes(C.byref(_paged(**kw))) == 0
    assert lib.ee_paged_bind(C.byref(_paged(**kw)), DUMMY, 1 << 60, C.byref(h)) == code
    assert not h.value


def _bound(**kw):
    lib, h, cfg = ee.load(), C.c_void_p(), _paged(**kw)
    n = lib.ee_paged_pool_bytes(C.byref(cfg))
    assert lib.ee_paged_bind(C.byref(cfg), DUMMY, n - 1, C.byref(h)) == ee.EE_ERR_CAPACITY
    assert lib.ee_paged_bind(C.byref(cfg), C.c_void_p(4097), n, C.byref(h)) == ee.EE_ERR_INVALID_ARG
    assert lib.ee_paged_bind(C.byref(cfg), None, n, C.byref(h)) == ee.EE_ERR_INVALID_ARG
    assert lib.ee_paged_bind(C.byref(cfg), DUMMY, n, C.byref(h)) == ee.EE_OK
    return lib, h


def test_pool_bytes():
    lib = ee.load()
    assert lib.ee_paged_pool_bytes(C.byref(_paged())) == 2 * 10 * 2 * 2 * 64 * 128 * 2
    assert lib.ee_paged_pool_bytes(C.byref(_paged(dtype=ee.EE_F32, head_dim=84))) == 2 * 10 * 2 * 2 * 64 * 84 * 4
    assert lib.ee_paged_pool_bytes(None) == 0


def _step(**kw):
    c = dict(n_seqs=2, n_tokens=3, max_q_len=2, max_kv_len=128, pages_per_seq=2, dev_q_start=4096, dev_kv_len=4096, dev_pages=4096,
             dev_status=None)
    c.update(kw)
    return ee.ee_paged_step(**c)


@pytest.mark.parametrize("kw,code", [
    (dict(n_seqs=-1), ee.EE_ERR_INVALID_ARG), (dict(n_tokens=-1), ee.EE_ERR_INVALID_ARG), (dict(max_kv_len=-1), ee.EE_ERR_INVALID_ARG),
    (dict(n_seqs=0), ee.EE_ERR_INVALID_ARG), (dict(max_q_len=0), ee.EE_ERR_INVALID_ARG), (dict(dev_pages=None), ee.EE_ERR_INVALID_ARG),
    (dict(dev_q_start=None), ee.EE_ERR_INVALID_ARG), (dict(dev_kv_len=None), ee.EE_ERR_INVALID_ARG),
    (dict(max_kv_len=129), ee.EE_ERR_CAPACITY), (dict(max_kv_len=2 ** 30 + 1, pages_per_seq=2 ** 30), ee.EE_ERR_CAPACITY),
])
def test_steps(kw, code):
    lib, p = _bound()
    heads = ee.ee_heads(4096, 256, 128)
    assert lib.ee_paged_append(p, 1, C.byref(_step(**kw)), None, C.byref(heads), C.byref(heads), None, None, 0, None) == code
    out = ee.ee_heads(8192, 256, 128)
    assert lib.ee_paged_attention(p, 1, C.byref(_step(**kw)), C.byref(heads), C.byref(out), 2, 1.0, 0, DUMMY, 1 << 50, None) == code
    lib.ee_paged_destroy(p)


def test_calls():
    lib, p = _bound()
    heads, out, none = ee.ee_heads(4096, 256, 128), ee.ee_heads(8192, 256, 128), ee.ee_heads(None, 256, 128)
    st, empty = C.byref(_step()), C.byref(_step(n_tokens=0))
    h, o, z = C.byref(heads), C.byref(out), C.byref(none)
    bad = ee.EE_ERR_INVALID_ARG
    assert lib.ee_paged_append(None, 1, st, None, h, h, None, None, 0, None) == bad
    assert lib.ee_paged_append(p, 1, None, None, h, h, None, None, 0, None) == bad
    assert lib.ee_paged_append(p, 0, st, None, h, h, None, None, 0, None) == ee.EE_ERR_LAYER_NOT_RESIDENT
    assert lib.ee_paged_append(p, 3, st, None, h, h, None, None, 0, None) == ee.EE_ERR_LAYER_NOT_RESIDENT
    assert lib.ee_paged_append(p, 1, st, None, h, None, None, None, 0, None) == bad
    assert lib.ee_paged_append(p, 1, st, None, h, z, None, None, 0, None) == bad
    assert lib.ee_paged_append(p, 1, st, None, h, h, None, None, 4, None) == bad
    assert lib.ee_paged_append(p, 1, st, None, h, h, h, o, -2, None) == bad
    assert lib.ee_paged_append(p, 1, st, None, h, h, h, o, 3, None) == ee.EE_ERR_SHAPE
    assert lib.ee_paged_append(p, 1, empty, None, None, None, None, None, 0, None) == ee.EE_OK
    wide = ee.ee_heads(4096, 512, 128)
    assert lib.ee_paged_append(p, 1, st, None, h, h, h, C.byref(wide), 2, None) == bad       # in place, other strides
    args = (DUMMY, 1 << 50, None)
    assert lib.ee_paged_attention(None, 1, st, h, o, 2, 1.0, 0, *args) == bad
    assert lib.ee_paged_attention(p, 1, st, h, o, 3, 1.0, 0, *args) == ee.EE_ERR_SHAPE
    assert lib.ee_paged_attention(p, 1, st, h, o, 0, 1.0, 0, *args) == ee.EE_ERR_SHAPE
    assert lib.ee_paged_attention(p, 1, st, h, o, 2, float("nan"), 0, *args) == bad
    assert lib.ee_paged_attention(p, 1, st, h, o, 2, 1.0, -1, *args) == bad
    assert lib.ee_paged_attention(p, 1, st, h, h, 2, 1.0, 0, *args) == bad
    assert lib.ee_paged_attention(p, 1, st, h, z, 2, 1.0, 0, *args) == bad
    assert lib.ee_paged_attention(p, 3, st, h, o, 2, 1.0, 0, *args) == ee.EE_ERR_LAYER_NOT_RESIDENT
    assert lib.ee_paged_attention(p, 1, empty, None, None, 2, 1.0, 0, None, 0, None) == ee.EE_OK
    need = lib.ee_paged_attention_workspace(p, 2, st)
    if need:
        assert lib.ee_paged_attention(p, 1, st, h, o, 2, 1.0, 0, DUMMY, need - 1, None) == ee.EE_ERR_CAPACITY
        assert lib.ee_paged_attention(p, 1, st, h, o, 2, 1.0, 0, None, need, None) == bad
        assert lib.ee_paged_attention(p, 1, st, h, o, 2, 1.0, 0, C.c_void_p(4097), need, None) == bad
    assert lib.ee_paged_attention_workspace(None, 2, st) == 0
    assert lib.ee_rope_apply(None, ee.EE_F32, h, o, DUMMY, 1, 1, 0, None, None) == bad
    assert lib.ee_paged_destroy(p) == ee.EE_OK and lib.ee_paged_destroy(None) == ee.EE_OK and lib.ee_rope_destroy(None) == ee.EE_OK


def test_the_workspace_grows_with_the_figures():
    """a workspace for some figures serves every step whose figures are smaller"""
    lib, p = _bound()
    base = dict(n_seqs=8, n_tokens=600, max_q_len=500, max_kv_len=4096, pages_per_seq=64)
    most = lib.ee_paged_attention_workspace(p, 16, C.byref(_step(**base)))
    for key in base:
        for v in (1, base[key] // 3, base[key] // 2, base[key] - 1):
            kw = dict(base, **{key: max(1, v)})
            kw["max_kv_len"] = min(kw["max_kv_len"], kw["pages_per_seq"] * 64)
            assert lib.ee_paged_attention_workspace(p, 16, C.byref(_step(**kw))) <= most, kw
    lib.ee_paged_destroy(p)
