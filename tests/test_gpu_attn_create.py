"""An attention context that cannot be made keeps nothing."""
import ctypes

import pytest
import torch

from paper_2607_13500_amd import _lib

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,allocations", [(_lib.TR_BF16, 5), (_lib.TR_FP32, 3)])
def test_create_reports_enomem_and_keeps_nothing(monkeypatch, dtype, allocations):
    """Each device allocation failing in turn gives TR_ENOMEM with *out == NULL and
    frees those before it (the attention's scratch among them, 68 MB)."""
    print("tr_attn_create allocation failures", dtype, flush=True)
    lib = _lib.load()
    p = _lib.AttnParams(heads=32, kv_heads=8, head_dim=128, rot_dim=128, axes=1, adjacent=0, dtype=dtype, norm=1, eps=1e-6, base=1e4)
    ctx = ctypes.c_void_p()
    # the process's first copy and fill set the runtime's own queues up (148 MB, once)
    assert lib.tr_attn_create(ctypes.byref(p), ctypes.byref(ctx)) == _lib.TR_OK
    lib.tr_attn_destroy(ctx)
    torch.cuda.synchronize()
    free0, _ = torch.cuda.mem_get_info()
    for k in range(1, allocations + 1):
        monkeypatch.setenv("TR_FAIL_ALLOC", str(k))
        for _ in range(4):
            ctx = ctypes.c_void_p(1234)
            assert lib.tr_attn_create(ctypes.byref(p), ctypes.byref(ctx)) == _lib.TR_ENOMEM, k
            assert ctx.value is None and b"failed" in lib.tr_last_error()
    monkeypatch.setenv("TR_FAIL_ALLOC", str(allocations + 1))      # there are no more
    for _ in range(4):
        assert lib.tr_attn_create(ctypes.byref(p), ctypes.byref(ctx)) == _lib.TR_OK and ctx.value
        lib.tr_attn_destroy(ctx)
    torch.cuda.synchronize()
    free1, _ = torch.cuda.mem_get_info()
    assert free0 - free1 < 32 << 20, (free0, free1)
