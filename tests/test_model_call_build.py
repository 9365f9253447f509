"""The native calls of a language model's worker: a module that is missing, damaged or made for another torch leaves the general calls, and is built again."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2106_05203_b200 import binding, build


def _changed(path, to):
    """A copy of the module that says it was built for another torch."""
    old = build.call_built_for().encode()
    data = open(binding.MODEL_CALL_PATH, "rb").read()
    assert data.count(old) >= 1
    open(path, "wb").write(data.replace(old, to.ljust(len(old))[:len(old)].encode()))


@pytest.mark.parametrize("kind", ["missing", "damaged", "another torch", "another module"])
def test_the_general_calls_are_left(kind, tmp_path):
    path = str(tmp_path / "_model_call.so")
    if kind == "damaged":
        open(path, "wb").write(b"no shared object")
    elif kind == "another torch":
        _changed(path, "torch 1.0")
    elif kind == "another module":
        shutil.copy(binding.CALL_PATH, path)
    with pytest.warns(RuntimeWarning, match="without their native calls"):
        calls = binding._load_model_calls(path)
    assert calls.embedding(torch.zeros(4, 4), torch.zeros(2), 1.0) is None and calls.policy_loss() is None


def test_the_module_that_fits_is_taken(recwarn):
    assert type(binding._load_model_calls()) is not binding._GeneralCalls and not [w for w in recwarn if "native call" in str(w.message)]


def test_entries_are_looked_at():
    with pytest.raises(TypeError):
        binding._model_calls.set_entries(1, 2)
    with pytest.raises(ValueError):
        binding._model_calls.set_entries(*[0] * 12)
    assert binding._model_calls.embedding() is None


def test_a_module_for_another_torch_or_header_is_built_again(tmp_path, monkeypatch):
    path, header, commands = str(tmp_path / "_model_call.so"), str(tmp_path / "ef21.h"), []

    def run(command, check):
        commands.append(command)
        open(command[command.index("-o") + 1], "w").close()
    monkeypatch.setattr(build, "MODEL_CALL", path)
    monkeypatch.setattr(build, "HEADER", header)
    monkeypatch.setattr(subprocess, "run", run)
    open(header, "w").close()
    shutil.copy(binding.MODEL_CALL_PATH, path)
    os.utime(path)
    build.build_model_call()
    assert commands == []
    _changed(path, "torch 1.0")
    build.build_model_call()
    assert len(commands) == 1
    shutil.copy(binding.MODEL_CALL_PATH, path)
    os.utime(path, (1, 1))
    build.build_model_call()
    assert len(commands) == 2
