"""The worker operators where the native module of their common calls is missing, broken or cannot be built, without a GPU."""
import importlib
import os
import subprocess
import sys
import warnings

import pytest
import torch

import paper_2010_04902_amd as B
from paper_2010_04902_amd import build, worker

NAME = "paper_2010_04902_amd._worker_calls"


@pytest.fixture
def unloaded(monkeypatch):
    worker._load()
    for name in ("_lib", "_calls"):
        monkeypatch.setattr(worker, name, None)
    monkeypatch.setitem(sys.modules, NAME, None)  # its import raises ModuleNotFoundError
    return monkeypatch


def _fails(error):
    def run(*args, **kw):
        raise error
    return run


ERRORS = [subprocess.CalledProcessError(1, ["g++"]), FileNotFoundError("g++"), PermissionError("read-only"), ImportError("no headers")]


@pytest.mark.parametrize("error", ERRORS, ids=lambda e: type(e).__name__)
def test_without_the_module_python_takes_every_call(unloaded, error):
    unloaded.setattr(build, "build_calls", _fails(error))
    x = torch.zeros(2, 8, 4, 4).contiguous(memory_format=torch.channels_last)
    with pytest.warns(RuntimeWarning, match="native module"):
        with pytest.raises(ValueError, match="CUDA"):  # the Python path's words
            B.byz_group_norm(x, 4)
    for name in ("group_norm", "group_norm_backward", "distill_loss", "distill_loss_step", "gated_ffn", "gated_ffn_backward"):
        assert getattr(worker._calls, name)(1, 2, 3) is None
    with warnings.catch_warnings():  # once
        warnings.simplefilter("error")
        with pytest.raises(ValueError, match="CUDA"):
            B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32))


def test_a_module_made_for_another_torch_is_built_again(unloaded):
    found, built = [], []

    def load(name, package=None):
        if not built:
            raise ImportError("undefined symbol")
        found.append(name)
        return "module"

    unloaded.setattr(worker.importlib, "import_module", load)
    unloaded.setattr(build, "build_calls", lambda: built.append(1))
    assert worker._load_calls() == "module" and built == [1] and len(found) == 1
    built.clear()
    unloaded.setattr(build, "build_calls", lambda: None)
    with pytest.warns(RuntimeWarning, match="undefined symbol"):
        assert isinstance(worker._load_calls(), worker._NoCalls)


def test_a_failed_build_leaves_no_old_module(tmp_path, monkeypatch):
    old = tmp_path / "_worker_calls.so"
    old.write_bytes(b"old")
    monkeypatch.setattr(build, "CALLS", str(old))
    monkeypatch.setattr(build.subprocess, "run", _fails(subprocess.CalledProcessError(1, ["g++"])))
    with pytest.raises(subprocess.CalledProcessError):
        build.build_calls()
    assert not old.exists() and not os.listdir(tmp_path)


def test_the_module_of_this_tree_is_there():
    assert importlib.import_module(NAME).group_norm() is None
