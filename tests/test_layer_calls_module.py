"""The extension module behind the operators around the recurrence: decode alone does not need it, it is looked for again after a failure, and
it is built for one torch.  No GPU."""
import ctypes
import os

import pytest
import torch

from paper_2609_33051_b200 import binding, build


class Stream:
    cuda_stream = 0


@pytest.fixture
def afresh(monkeypatch):
    """A process that has loaded nothing yet."""
    build.build()
    monkeypatch.setattr(binding, "_LIB", None)
    monkeypatch.setattr(binding, "_CALLS", None)
    return monkeypatch


def test_decode_alone_needs_no_extension_module(afresh, tmp_path):
    afresh.setattr(build, "calls_path", lambda: str(tmp_path / "none.so"))
    for _ in range(2):
        lib = binding.load_library()
        m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, device=0, allocate=False)
        n = ctypes.c_size_t()
        assert lib.sketchssm_prompt_work_bytes(m._ctx, 1, 1, ctypes.byref(n)) == 0
        with pytest.raises(FileNotFoundError, match="none.so not found: build it with"):
            m.rms_norm(torch.zeros(1, 8), torch.zeros(8), stream=Stream)
    afresh.undo()
    with pytest.raises(ValueError, match="x is a Float tensor"):
        m.rms_norm(torch.zeros(1, 8), torch.zeros(8), stream=Stream)


def test_a_module_that_does_not_load_is_tried_again(afresh, tmp_path):
    bad = tmp_path / "bad.so"
    bad.write_bytes(b"no library")
    with afresh.context() as c:
        c.setattr(build, "calls_path", lambda: str(bad))
        m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, device=0, allocate=False)
        for _ in range(2):
            with pytest.raises(ImportError):
                m.rms_norm(torch.zeros(1, 8), torch.zeros(8), stream=Stream)
    with pytest.raises(ValueError, match="x is a Float tensor"):
        m.rms_norm(torch.zeros(1, 8), torch.zeros(8), stream=Stream)


def test_the_module_is_built_for_one_torch(monkeypatch):
    """Another torch asks for another file, so that a module of the old one is neither kept by the build nor loaded."""
    build.build()
    mine = build.calls_path()
    assert os.path.exists(mine) and torch.__version__ in os.path.basename(mine)
    monkeypatch.setattr(torch, "__version__", "2.99.0")
    other = build.calls_path()
    assert other != mine and other in build._calls_command() and not os.path.exists(other)
    monkeypatch.setattr(binding, "_CALLS", None)
    m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, device=0, allocate=False)
    with pytest.raises(FileNotFoundError, match="2.99.0"):
        m.rms_norm(torch.zeros(1, 8), torch.zeros(8), stream=Stream)
