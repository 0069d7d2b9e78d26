"""Host-side checks of the lookup's, the layer norm's and AdamW's entry points (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_1410_8043_gb300 import build

    lib = ctypes.CDLL(build.build())
    for name in ("embed", "norm", "adamw"):
        getattr(lib, f"esspt_{name}_workspace_bytes").restype = ctypes.c_size_t
        getattr(lib, f"esspt_{name}_last_error").restype = ctypes.c_char_p
    lib.esspt_adamw_moment_values.restype = ctypes.c_int64
    return lib


@pytest.mark.parametrize("c, py", [("esspt_embed_config", "EmbedConfig"), ("esspt_norm_config", "NormConfig"),
                                   ("esspt_adamw_config", "AdamWConfig"), ("esspt_adamw_tensor", "AdamWTensor")])
def test_layouts_match_c(tmp_path, c, py):
    from paper_1410_8043_gb300 import esspt

    S = getattr(esspt, py)
    names = [f[0] for f in S._fields_]
    probe = tmp_path / "probe.c"
    probe.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "esspt.h"\nint main(void){printf("%zu"'
                     + "".join(' " %zu"' for _ in names) + f", sizeof({c})"
                     + "".join(f", offsetof({c}, {n})" for n in names) + ");return 0;}\n")
    exe = tmp_path / "probe"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(probe), "-o", str(exe)])
    got = list(map(int, subprocess.check_output([str(exe)]).split()))
    assert got == [ctypes.sizeof(S)] + [getattr(S, n).offset for n in names]


def test_embed_configurations(L):
    from paper_1410_8043_gb300 import esspt

    def size(**kw):
        c = dict(max_tokens=8, n_rows=1000, width=64, dtype=0, backward=1, **{})
        c.update(kw)
        cfg = esspt.EmbedConfig(c["max_tokens"], c["n_rows"], c["width"], c["dtype"], c["backward"], None)
        bytes_ = L.esspt_embed_workspace_bytes(ctypes.byref(cfg))
        if bytes_ == 0:  # create refuses what the size query refuses
            h = ctypes.c_void_p()
            assert L.esspt_embed_create(ctypes.byref(cfg), ctypes.c_void_p(256), ctypes.c_size_t(1 << 40), ctypes.byref(h)) == 1
            assert L.esspt_embed_last_error(None) != b""
        return bytes_

    assert size() > 0 and size(backward=0) <= size() and size(max_tokens=1 << 20) > size()
    assert size(max_tokens=1 << 30, n_rows=1 << 30, width=8192) > 0
    for bad in (dict(max_tokens=0), dict(max_tokens=(1 << 30) + 1), dict(n_rows=0), dict(n_rows=(1 << 30) + 1), dict(width=0),
                dict(width=8193), dict(dtype=3), dict(dtype=-1)):
        assert size(**bad) == 0, bad
    assert L.esspt_embed_workspace_bytes(None) == 0


def test_norm_configurations(L):
    from paper_1410_8043_gb300 import esspt

    def size(**kw):
        c = dict(max_rows=8, width=64, dtype=1, weight_dtype=0, backward=1, eps=1e-5)
        c.update(kw)
        cfg = esspt.NormConfig(c["max_rows"], c["width"], c["dtype"], c["weight_dtype"], c["backward"], c["eps"], None)
        bytes_ = L.esspt_norm_workspace_bytes(ctypes.byref(cfg))
        if bytes_ == 0:
            h = ctypes.c_void_p()
            assert L.esspt_norm_create(ctypes.byref(cfg), ctypes.c_void_p(256), ctypes.c_size_t(1 << 40), ctypes.byref(h)) == 1
            assert L.esspt_norm_last_error(None) != b""
        return bytes_

    assert size() > 0 and size(backward=0) <= size() and size(weight_dtype=1) > 0
    for bad in (dict(max_rows=0), dict(max_rows=1 << 31), dict(width=0), dict(width=8193), dict(dtype=3), dict(weight_dtype=2),
                dict(dtype=0, weight_dtype=1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert size(**bad) == 0, bad
    assert L.esspt_norm_workspace_bytes(None) == 0


def test_adamw_configurations(L):
    from paper_1410_8043_gb300 import esspt

    def size(counts=(5, 0, 300), decay=0.01, **kw):
        c = dict(n=len(counts), bits=32, copy=1, reserved=0, b1=0.9, b2=0.999, eps=1e-8)
        c.update(kw)
        recs = (esspt.AdamWTensor * max(1, len(counts)))(*[esspt.AdamWTensor(256 if n else None, None, n, decay) for n in counts])
        cfg = esspt.AdamWConfig(c["n"], c["bits"], c["copy"], c["reserved"], c["b1"], c["b2"], c["eps"], 0, None)
        bytes_ = L.esspt_adamw_workspace_bytes(ctypes.byref(cfg), recs)
        values = L.esspt_adamw_moment_values(ctypes.byref(cfg), recs)
        if bytes_ == 0:
            h = ctypes.c_void_p()
            assert values == 0
            assert L.esspt_adamw_create(ctypes.byref(cfg), recs, ctypes.c_void_p(256), ctypes.c_size_t(1 << 40), ctypes.byref(h)) == 1
            assert L.esspt_adamw_last_error(None) != b""
        else:
            assert values == sum(-(-n // 128) * 128 for n in counts)
        return bytes_

    assert size() >= 512 * 8 and size(bits=8) > 0
    assert size(counts=(1 << 20,), bits=8) < size(counts=(1 << 20,)) / 3
    for bad in (dict(n=0), dict(n=(1 << 20) + 1), dict(bits=16), dict(copy=0), dict(copy=3), dict(reserved=1), dict(b1=1.0),
                dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(eps=0.0), dict(eps=1e-60), dict(eps=float("inf")),
                dict(counts=(-1,)), dict(decay=-1.0), dict(decay=float("nan"))):
        assert size(**bad) == 0, bad
    assert L.esspt_adamw_workspace_bytes(None, None) == 0


def test_null_handles(L):
    null = ctypes.c_void_p()
    for name in ("embed", "norm", "adamw"):
        assert getattr(L, f"esspt_{name}_destroy")(null) == 0
    assert L.esspt_embed_poll(null) == 1 and L.esspt_adamw_steps(null, null) == 1
    assert L.esspt_adamw_moments(null, null, null) == 1


def test_no_gpu_means_no_handles():
    from paper_1410_8043_gb300 import esspt

    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        esspt.Embedding(4, 10, 8)
    with pytest.raises(RuntimeError):
        esspt.LayerNorm(4, 8)
    with pytest.raises(RuntimeError):
        esspt.AdamW([torch.zeros(4)])


@pytest.mark.parametrize("tensors, wrong", [
    ([(4096, 0, 100), (4096, 0, 100)], True), ([(4096, 0, 100), (4492, 0, 10)], True), ([(4492, 0, 10), (4096, 0, 100)], True),
    ([(4096, 4400, 100)], True), ([(4096, 8192, 100), (8392, 0, 5), (8388, 0, 0)], False), ([(4096, 8192, 100), (8388, 0, 5)], True),
    ([(4096, 8192, 100), (16384, 8390, 3)], True), ([(4096, 0, 100), (4496, 0, 10)], False), ([(0, 0, 0), (0, 0, 0), (4096, 0, 1)], False),
    ([(4096, 0, 0), (4096, 0, 7)], False)])
def test_adamw_refuses_tensors_that_overlap(L, tensors, wrong):
    """The same parameter twice, or parts of it: blocks would write it at the same time.  Empty ones are nowhere."""
    from paper_1410_8043_gb300 import esspt

    recs = (esspt.AdamWTensor * len(tensors))(*[esspt.AdamWTensor(p or None, c or None, n, 0.0) for p, c, n in tensors])
    cfg = esspt.AdamWConfig(len(tensors), 32, 1, 0, 0.9, 0.999, 1e-8, 0, None)
    need, h = L.esspt_adamw_workspace_bytes(ctypes.byref(cfg), recs), ctypes.c_void_p()
    # (one byte too few where nothing overlaps: refused for that, and nothing is made of these addresses)
    st = L.esspt_adamw_create(ctypes.byref(cfg), recs, ctypes.c_void_p(1 << 30), ctypes.c_size_t(need if wrong else need - 1), ctypes.byref(h))
    assert (st == esspt.EINVAL and b"overlap" in L.esspt_adamw_last_error(None)) if wrong else st == esspt.ENOSPC


def test_waits_are_for_the_handles_device(monkeypatch):
    """Polls, step counts and the end are called with the handle's device current: its default stream is that device's."""
    from paper_1410_8043_gb300 import esspt

    current, seen = ["cuda:0"], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            current.append(self.device)

        def __exit__(self, *exc):
            current.pop()

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, current[-1])) or 0

    monkeypatch.setattr(esspt.torch.cuda, "device", Device)
    em, aw = esspt.Embedding.__new__(esspt.Embedding), esspt.AdamW.__new__(esspt.AdamW)
    for handle in (em, aw):
        handle._lib, handle._h, handle.device = Library(), 1, "cuda:1"
    em.poll()
    assert aw.steps == 0
    em.close(), aw.close(), aw.close()
    assert seen == [(f"esspt_{name}", "cuda:1") for name in ("embed_poll", "adamw_steps", "embed_destroy", "adamw_destroy")]
