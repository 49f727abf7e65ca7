"""What is built from what (nothing is compiled here)."""
import sys
import types

import pytest


@pytest.fixture
def steps(monkeypatch):
    """The commands that a build starts; those that name `steps.broken` fail."""
    from oracle import build as oracle_build
    from paper_2110_10548_amd import binding, build
    seen = types.SimpleNamespace(build=build, commands=[], broken=None)

    def start(cmd, **_):
        seen.commands.append(cmd)
        rc = int(seen.broken is not None and any(seen.broken in c for c in cmd))
        return types.SimpleNamespace(wait=lambda: rc, returncode=rc)

    monkeypatch.setattr(build.subprocess, "Popen", start)
    monkeypatch.setattr(build.subprocess, "run", start)
    monkeypatch.setattr(oracle_build, "build", lambda force: seen.commands.append(["oracle"]))
    monkeypatch.setattr(binding, "lib", lambda: seen.commands.append(["loaded"]))
    return seen


def outputs(steps):
    return [c[c.index("-o") + 1].rsplit("/", 1)[1] if "-o" in c else c[0] for c in steps.commands if "-c" not in c]


def test_the_library_is_built_without_torch(steps, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)       # (importing it fails)
    steps.build.build()
    assert outputs(steps) == ["libp2.so"] and all(c[0] == "hipcc" for c in steps.commands)
    assert len(steps.commands) == len(steps.build.SOURCES) + 1


def test_everything_is_built_without_torch_but_its_module(steps, monkeypatch, capsys):
    import __graft_entry__
    monkeypatch.setitem(sys.modules, "torch", None)
    __graft_entry__.build()
    assert outputs(steps) == ["libp2.so", "oracle", "loaded"] and "torch is not installed" in capsys.readouterr().out


def test_a_module_that_does_not_compile_is_an_error_once_the_library_is_there(steps):
    import __graft_entry__
    steps.broken = "p2_train_tensors.cpp"
    with pytest.raises(RuntimeError, match="p2_train_tensors"):
        __graft_entry__.build()
    assert outputs(steps) == ["libp2.so", "oracle", "loaded", "_train.so"]
