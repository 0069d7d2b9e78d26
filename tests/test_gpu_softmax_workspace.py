"""A handle writes within the bytes of workspace it asked for, and only there (GPU)."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,max_top,top", [
    (8, 3000, 5, 1, 1), (97, 1000, 16, 3, 3), (100, 40_001, 8, 1, 1), (200, 300, 1, 1, 1), (100_000, 200, 1, 1, 1), (9000, 500, 2, 4, 1),
    (3000, 2000, 7, 2, 2), (300, 60_001, 130, 5, 5), (700, 1500, 500, 1, 1), (400, 900, 64, 300, 300), (2000, 129, 33, 17, 9)])
def test_writes_stay_inside(T, V, D, max_top, top, dtype):
    from paper_1410_8043_gb300 import esspt

    kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    L = esspt.lib()
    stream = torch.cuda.current_stream().cuda_stream
    cfg = esspt.SoftmaxConfig(T, V, D, esspt.DTYPES[kind], max_top, 1, ctypes.c_void_p(stream))
    need = L.esspt_softmax_workspace_bytes(ctypes.byref(cfg))
    assert need > 0
    mem = torch.full((GUARD + need + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    at = mem.data_ptr() + GUARD
    assert at % 256 == 0
    h = ctypes.c_void_p()
    assert L.esspt_softmax_create(ctypes.byref(cfg), at, need, ctypes.byref(h)) == esspt.OK
    g = torch.Generator("cuda").manual_seed(T)
    x = (torch.randn((T, D), generator=g, device="cuda")).to(kind)
    w = (torch.randn((V, D), generator=g, device="cuda")).to(kind)
    ids = torch.randint(0, V, (T, top), generator=g, device="cuda").int()
    z = torch.randn((T, top), generator=g, device="cuda")
    out = [torch.zeros(T, device="cuda") for _ in range(2)] + [torch.zeros_like(x), torch.zeros_like(w)]
    ptr = [o.data_ptr() for o in out]
    for n in (T, max(1, T // 3), min(T, 8)):
        for grads in (ptr[2:], [None, None]):
            tail = (n, None, 1.0, *ptr[:2], *grads)
            assert L.esspt_softmax_loss(h, x.data_ptr(), D, w.data_ptr(), D, ids.data_ptr(), *tail) == esspt.OK
            assert L.esspt_softmax_distill(h, x.data_ptr(), D, w.data_ptr(), D, ids.data_ptr(), z.data_ptr(), top, *tail) == esspt.OK
    assert L.esspt_softmax_poll(h) == esspt.OK and L.esspt_softmax_destroy(h) == esspt.OK
    assert bool((mem[:GUARD] == 0xA5).all()) and bool((mem[GUARD + need:] == 0xA5).all())
    assert all(bool(torch.isfinite(o).all()) for o in out)
