"""_bpt_torch.so is compiled against one PyTorch and one Python: the key inside it decides, beside the files' times, whether it is
built again, and whether it is loaded.  No GPU needed."""
import os
import shutil

import pytest


@pytest.fixture
def lib(tmp_path, monkeypatch):
    from paper_1911_04070_b200 import binding, build
    build.build()
    at = str(tmp_path / "_bpt_torch.so")
    shutil.copy(build.LIB_TORCH, at)
    monkeypatch.setattr(build, "LIB_TORCH", at)
    monkeypatch.setattr(binding, "_native", None)
    started = []
    monkeypatch.setattr(build.subprocess, "Popen", lambda cmd: started.append(cmd))
    return build, binding, at, started


def _put(at, change):
    data = open(at, "rb").read()
    with open(at, "wb") as f:
        f.write(change(data))


def test_the_key_is_read_from_the_file(lib):
    build, binding, at, started = lib
    assert build.built_for(at) == build.torch_key()
    assert build.built_for(at + ".none") is None
    assert build._start_torch(False) is None and not started        # up to date
    assert build._start_torch(True) is not None and len(started) == 1


@pytest.mark.parametrize("change", [lambda d: d.replace(b"BPT_TORCH_KEY:torch ", b"BPT_TORCH_KEY:tOrch "), lambda d: d.replace(b"BPT_TORCH_KEY:", b"BPT_TORCH_xxx:"),
                                    lambda d: b""])
def test_a_file_of_another_pytorch_is_built_again_and_not_loaded(lib, change):
    build, binding, at, started = lib
    _put(at, change)
    assert os.path.getmtime(at) >= os.path.getmtime(build.SRC_TORCH)      # as new as its sources: the time alone would keep it
    with pytest.raises(ImportError, match="build"):
        binding.load_native()
    assert build._start_torch(False) is not None and len(started) == 1


def test_the_built_file_is_loaded():
    from paper_1911_04070_b200 import binding
    assert binding.load_native() is not None
