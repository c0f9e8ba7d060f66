"""The build and the binding's shortcut (CPU): libgraphleap.so does not depend on
_calls.so, neither when it is built nor when its calls are made."""
import os
import sys

import pytest
import torch

import paper_2604_21290_amd as pkg
from paper_2604_21290_amd import api, build


@pytest.fixture
def fake(tmp_path, monkeypatch):
    """build_library with compilers that only write their outputs; `bad` names the
    sources that they fail on."""
    bad = set()

    def run(cmd):
        for name in bad:
            if any(os.path.basename(c) == name for c in cmd):
                return 1, f"cannot compile {name}"
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")
        return 0, ""

    (tmp_path / "_build").mkdir()
    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(build, "ROOT", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    return bad


def test_build_makes_both(fake):
    assert build.build_library(verbose=False) == build.LIB
    assert os.path.exists(build.LIB) and os.path.exists(build.CALLS)


def test_library_is_linked_where_the_shortcut_does_not_compile(fake):
    with open(build.CALLS, "w") as f:
        f.write("an older one")
    fake.add("calls.cpp")
    with pytest.raises(RuntimeError, match="complete, but not the binding's shortcut") as e:
        build.build_library(verbose=False)
    assert "cannot compile calls.cpp" in str(e.value.__cause__)
    assert os.path.exists(build.LIB) and not os.path.exists(build.CALLS)


def test_hipcc_errors_are_told_first(fake):
    fake |= {"calls.cpp", "norm.hip"}
    with pytest.raises(RuntimeError, match="hipcc failed .*\n?.*norm.hip"):
        build.build_library(verbose=False)
    assert not os.path.exists(build.LIB)


@pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libgraphleap.so not built")
def test_calls_without_the_shortcut(monkeypatch):
    monkeypatch.setattr(api, "_native", None)
    monkeypatch.delattr(pkg, "_calls", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2604_21290_amd._calls", None)
    x = torch.zeros(4, 64)
    with pytest.warns(RuntimeWarning, match="_calls.so cannot be loaded"):
        n = api._calls()
    # every form is left to the Python path, whose own check this is
    for f, args in ((n.layer_norm, (x, None, None, 1e-5, False)), (n.layer_norm_backward, (x, x, x, x, None)),
                    (n.quantize_rows, (x,)), (n.layer_norm_q8, (x, None, None, 1e-5)), (n.linear_q8, (x,) * 10)):
        assert f(*args) is None
    for call in (api.layer_norm, api.quantize_rows, api.layer_norm_q8):
        with pytest.raises(ValueError, match="device tensor"):
            call(x)
