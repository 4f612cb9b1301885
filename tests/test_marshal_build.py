"""The marshalling module and the library are built, found and copied as a program's tree changes: no GPU."""
import copy
import dataclasses
import os
import pickle

import pytest
import torch

from paper_2511_05534_b200 import binding as F
from paper_2511_05534_b200 import build


def test_a_module_of_another_torch_or_interpreter_is_not_loaded(monkeypatch):
    """It knows where torch's and Python's objects have their fields: one that was built for others would read addresses from elsewhere."""
    build.build()
    F._load_marshal()
    here = build.marshal_path()
    assert os.path.exists(here)
    for change in (lambda m: m.setattr(torch, "__version__", "0.0.0+other"), lambda m: m.setattr("sysconfig.get_config_var", lambda name: "cpython-39-other")):
        with monkeypatch.context() as m:
            change(m)
            m.setattr(F, "_marshal", None)
            assert build.marshal_path() != here and not os.path.exists(build.marshal_path())
            with pytest.raises(FileNotFoundError, match="build"):
                F._load_marshal()


def test_the_library_is_built_without_what_the_module_needs(monkeypatch, tmp_path):
    """No g++, no headers of Python or torch: the C library is there all the same, and the build says what is missing."""
    commands = []

    def run(command, *args, **kwargs):
        commands.append(command[0])
        if command[0] != "nvcc":
            raise FileNotFoundError(command[0])
        open(command[command.index("-o") + 1], "w").close()
    monkeypatch.setattr(build.subprocess, "check_call", run)
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "libflowmm.so"))
    monkeypatch.setattr(build, "marshal_path", lambda: str(tmp_path / "_marshal.so"))
    with pytest.raises(FileNotFoundError, match="g\\+\\+"):
        build.build(force=True)
    assert commands == ["nvcc", "g++"] and os.path.exists(build.LIB_PATH) and not os.path.exists(build.marshal_path())


def test_params_are_copied_and_sent_on_after_a_call():
    """What a call leaves in them is an address of this process and of these fields: copies begin without it."""
    build.build()
    p = F.CacheParams(2, 8, 2, 128, 64, 10, 4, 8, softmax_scale=0.5)
    F._cache_call(p, "flowmm_cache_plan")
    assert p.calls
    for q in (copy.copy(p), copy.deepcopy(p), pickle.loads(pickle.dumps(p)), dataclasses.replace(p)):
        assert q == p and not q.calls and p.calls
        q.n_rows = 3
        F._cache_call(q, "flowmm_cache_plan")
        assert p.n_rows == 8 and q.calls != p.calls
    assert p.calls
    p.n_rows = 3
    assert not p.calls
