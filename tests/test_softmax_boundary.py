"""Host-side checks of the softmax entry points (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_config_layout_matches_c(tmp_path):
    from paper_1410_8043_gb300 import esspt

    names = [f[0] for f in esspt.SoftmaxConfig._fields_]
    probe = tmp_path / "probe.c"
    probe.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "esspt.h"\nint main(void){printf("%zu"'
                     + "".join(' " %zu"' for _ in names) + ', sizeof(esspt_softmax_config)'
                     + "".join(f", offsetof(esspt_softmax_config, {n})" for n in names) + ");return 0;}\n")
    exe = tmp_path / "probe"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(probe), "-o", str(exe)])
    got = list(map(int, subprocess.check_output([str(exe)]).split()))
    assert got == [ctypes.sizeof(esspt.SoftmaxConfig)] + [getattr(esspt.SoftmaxConfig, n).offset for n in names]


def test_dtypes_and_limits_match_the_header():
    import torch

    from paper_1410_8043_gb300 import esspt

    src = open(os.path.join(ROOT, "include", "esspt.h")).read()
    for dtype, name in ((torch.float32, "ESSPT_F32"), (torch.bfloat16, "ESSPT_BF16"), (torch.float16, "ESSPT_F16")):
        assert f"{name} = {esspt.DTYPES[dtype]}" in src


def test_invalid_configurations_have_no_workspace():
    """The size query refuses what create refuses, and a narrower handle needs less."""
    import torch  # noqa: F401  (loads the CUDA runtime the library links against)

    from paper_1410_8043_gb300 import build, esspt

    L = ctypes.CDLL(build.build())
    L.esspt_softmax_workspace_bytes.restype = ctypes.c_size_t

    def size(**kw):
        c = dict(max_rows=8, n_items=1000, width=64, dtype=0, max_top=1, backward=1)
        c.update(kw)
        cfg = esspt.SoftmaxConfig(c["max_rows"], c["n_items"], c["width"], c["dtype"], c["max_top"], c["backward"], None)
        return L.esspt_softmax_workspace_bytes(ctypes.byref(cfg))

    assert size() > 0 and size(backward=0) < size()
    for bad in (dict(max_rows=0), dict(max_rows=(1 << 20) + 1), dict(n_items=0), dict(n_items=(1 << 30) + 1), dict(width=0),
                dict(width=513), dict(dtype=3), dict(dtype=-1), dict(max_top=0), dict(max_rows=1 << 20, max_top=2048)):
        assert size(**bad) == 0, bad
    assert L.esspt_softmax_workspace_bytes(None) == 0


def test_no_gpu_means_no_head():
    import torch

    from paper_1410_8043_gb300 import esspt

    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        esspt.SoftmaxHead(4, 10, 8)
