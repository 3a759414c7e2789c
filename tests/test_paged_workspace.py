"""The attention's workspace, without a GPU: what is refused, for calls that need one."""
import ctypes as C

import pytest

from paper_2504_10724_amd import capi as ee

DUMMY = C.c_void_p(4096)


@pytest.mark.parametrize("dtype,hd", [(ee.EE_BF16, 128), (ee.EE_BF16, 256), (ee.EE_F32, 64), (ee.EE_F32, 200)])
@pytest.mark.parametrize("rows", [1, 500])
def test_workspaces_that_do_not_do_are_refused(dtype, hd, rows):
    lib, p = ee.load(), C.c_void_p()
    cfg = ee.ee_paged_config(2, 10, 2, hd, 64, dtype)
    assert lib.ee_paged_bind(C.byref(cfg), DUMMY, lib.ee_paged_pool_bytes(C.byref(cfg)), C.byref(p)) == ee.EE_OK
    st = C.byref(ee.ee_paged_step(2, rows + 1, rows, 4096, 64, 4096, 4096, 4096, None))
    q, out = C.byref(ee.ee_heads(4096, 4 * hd, hd)), C.byref(ee.ee_heads(8192, 4 * hd, hd))
    need = lib.ee_paged_attention_workspace(p, 4, st)
    assert need > 0 and need % 4 == 0
    call = lambda ws, n: lib.ee_paged_attention(p, 1, st, q, out, 4, 1.0, 0, ws, n, None)      # noqa: E731
    assert call(DUMMY, need - 1) == ee.EE_ERR_CAPACITY and call(DUMMY, 0) == ee.EE_ERR_CAPACITY
    assert call(None, need) == ee.EE_ERR_INVALID_ARG
    assert call(C.c_void_p(4097), need) == ee.EE_ERR_INVALID_ARG
    assert call(C.c_void_p(4096 + 128), need) == ee.EE_ERR_INVALID_ARG
    # the handle's and the figures' own faults
    for n_q, step in ((3, st), (0, st), (-2, st), (4, C.byref(ee.ee_paged_step(0, 0, 0, 4096, 64, 4096, 4096, 4096, None)))):
        assert lib.ee_paged_attention_workspace(p, n_q, step) == 0
    assert lib.ee_paged_attention_workspace(p, 4, None) == 0
    lib.ee_paged_destroy(p)
