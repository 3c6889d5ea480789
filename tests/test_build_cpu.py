"""The build of the library and of the sequence operators' binding, its commands replaced by records of them."""
import os
import types

import pytest

torch = pytest.importorskip("torch")
from paper_1902_11208_amd import build  # noqa: E402


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """Paths in tmp_path; a command that has run wrote its -o file. commands.fail: a name whose command fails."""
    done = types.SimpleNamespace(list=[], fail=None)

    def run(cmd, **kw):
        done.list.append(cmd)
        bad = done.fail is not None and any(done.fail in c for c in cmd)
        if not bad:
            open(cmd[cmd.index("-o") + 1], "w").write("new")
        return types.SimpleNamespace(returncode=int(bad), stdout="", stderr="")

    monkeypatch.setattr(build, "subprocess", types.SimpleNamespace(run=run))
    for name in ("BUILD", "LIB", "BINDING"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    return done


def test_library_does_not_need_the_binding(commands):
    open(build.BINDING, "w").write("old")
    commands.fail = "binding.cpp"
    with pytest.raises(RuntimeError, match="libmdlstm.so is built"):
        build.build()
    assert open(build.LIB).read() == "new"
    assert not os.path.exists(build.BINDING), "a binding of an earlier build beside a new library"
    commands.fail = None
    assert build.build() == build.LIB
    assert open(build.BINDING).read() == "new"


@pytest.mark.parametrize("new_abi", [False, True])
def test_binding_has_the_string_layout_of_torch(commands, monkeypatch, new_abi):
    monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: new_abi)
    build.build()
    cmd = next(c for c in commands.list if any("binding.cpp" in x for x in c))
    assert [x for x in cmd if "CXX11_ABI" in x] == [f"-D_GLIBCXX_USE_CXX11_ABI={int(new_abi)}"]
