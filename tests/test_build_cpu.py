"""When the build compiles again."""
import os
import time

import torch

from paper_2509_24899_b200 import build


def test_the_module_of_the_torch_calls_is_stale_for_another_pytorch(monkeypatch, tmp_path):
    build.build()
    assert not build._torch_calls_stale()
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".other")
    assert build._torch_calls_stale()
    monkeypatch.undo()
    assert not build._torch_calls_stale()
    monkeypatch.setattr(build, "BUILT_FOR", str(tmp_path / "nothing"))        # made by a build that did not say for what
    assert build._torch_calls_stale()


def test_the_module_is_compiled_again_for_another_pytorch(monkeypatch, tmp_path):
    """With a compiler that only notes that it was called."""
    log, cxx = tmp_path / "called", tmp_path / "cxx"
    cxx.write_text('#!/bin/sh\necho "$@" >> %s\n' % log)
    cxx.chmod(0o755)
    build.build()
    stamp = tmp_path / "as_torch_calls.so.built_for"
    stamp.write_text(build.torch_key())
    monkeypatch.setattr(build, "BUILT_FOR", str(stamp))
    monkeypatch.setenv("CXX", str(cxx))
    before = os.path.getmtime(build.TORCH_CALLS)
    build.build_torch_calls()
    assert not log.exists()
    stamp.write_text("torch 0.0, python 0.0")
    build.build_torch_calls()
    assert log.read_text().count("torch_calls.cpp") == 1 and stamp.read_text() == build.torch_key()
    build.build_torch_calls()
    assert log.read_text().count("torch_calls.cpp") == 1
    assert os.path.getmtime(build.TORCH_CALLS) == before <= time.time()
