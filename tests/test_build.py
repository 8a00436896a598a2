"""What build.py makes, and when: with compilers that only note what they were asked for."""
import importlib.util
import os
import shutil
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent

COMPILER = """#!/bin/sh
echo "$0 $*" >> LOG
[ -f LOG.fail ] && exit 1
src=
while [ $# -gt 0 ]; do
    case "$1" in
        -o) out=$2; shift ;;
        -MF) deps=$2; shift ;;
        *.cu) src=$1 ;;
    esac
    shift
done
[ -n "$deps" ] && echo "x.o: $src" > "$deps"
echo made > "$out"
"""


class Tree:
    def __init__(self, root: Path, monkeypatch):
        self.root, self.monkeypatch = root, monkeypatch
        pkg = root / "pkg"
        for d in (pkg / "csrc", root / "include", root / "torch"):
            d.mkdir(parents=True)
        for f in ("api.cu", "serve.cu", "common.cuh", "host_state.h", "torch_binding.cpp"):
            (pkg / "csrc" / f).write_text("")
        (root / "include" / "mmv.h").write_text("")
        (root / "torch" / "version.py").write_text("__version__ = '1'")
        for name in ("nvcc", "cxx"):
            c = root / "bin" / name
            c.parent.mkdir(exist_ok=True)
            c.write_text(COMPILER.replace("LOG", str(root / f"{name}.log")))
            c.chmod(0o755)
        monkeypatch.setenv("NVCC", str(root / "bin" / "nvcc"))
        monkeypatch.setenv("CXX", str(root / "bin" / "cxx"))
        monkeypatch.delenv("MMV_NVCC_FLAGS", raising=False)
        (pkg / "build.py").write_text((ROOT / "paper_2506_23906_b200" / "build.py").read_text())
        spec = importlib.util.spec_from_file_location("_build_under_test", pkg / "build.py")
        self.mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(self.mod)
        find = importlib.util.find_spec
        found = importlib.util.spec_from_file_location("torch", root / "torch" / "__init__.py")
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: found if name == "torch" else find(name, *a))
        self.age()

    def age(self):
        """Everything that is there becomes older than what is written next."""
        for f in self.root.rglob("*"):
            if f.is_file():
                t = f.stat().st_mtime - 100
                os.utime(f, (t, t))

    def touch(self, name):
        os.utime(self.root / name)

    def ran(self):
        """The compilers' calls since the last time that this was asked: (sources compiled, libraries linked, extensions)."""
        logs = [self.root / f"{n}.log" for n in ("nvcc", "cxx")]
        nvcc, cxx = (p.read_text().splitlines() if p.exists() else [] for p in logs)
        for p in logs:
            p.unlink(missing_ok=True)
        return sorted(Path(c.split()[-1]).name for c in nvcc if " -c " in c), sum(" -c " not in c for c in nvcc), len(cxx), nvcc

    def build(self, **how):
        self.mod.build(**how)
        self.age()
        return self.ran()


@pytest.fixture
def tree(tmp_path, monkeypatch):
    return Tree(tmp_path, monkeypatch)


def test_everything_once(tree):
    assert tree.build()[:3] == (["api.cu", "serve.cu"], 1, 1)
    assert tree.build()[:3] == ([], 0, 0)
    assert tree.build(force=True)[:3] == (["api.cu", "serve.cu"], 1, 1)


def test_a_source_compiles_alone(tree):
    tree.build()
    tree.touch("pkg/csrc/serve.cu")
    assert tree.build()[:3] == (["serve.cu"], 1, 0)
    tree.touch("pkg/csrc/torch_binding.cpp")
    assert tree.build()[:3] == ([], 0, 1)


def test_another_torch_compiles_the_extension(tree):
    tree.build()
    (tree.root / "torch" / "version.py").write_text("__version__ = '2'")
    tree.age()
    assert tree.mod.needs_build() and tree.build()[:3] == ([], 0, 1)
    assert not tree.mod.needs_build()


def test_a_failed_extension_is_made_again(tree):
    """Against a header that changed, the extension fails to compile behind a library that did: the next build makes it."""
    tree.build()
    tree.touch("include/mmv.h")
    (tree.root / "cxx.log.fail").write_text("")
    with pytest.raises(Exception):
        tree.mod.build()
    (tree.root / "cxx.log.fail").unlink()
    tree.ran()
    assert tree.build()[2] == 1


def test_other_flags_compile_every_object(tree):
    """A library that is built at all is built whole with the flags of that build."""
    tree.build()
    tree.monkeypatch.setenv("MMV_NVCC_FLAGS", "-DOTHER")
    tree.touch("pkg/csrc/serve.cu")
    sources, links, _, calls = tree.build()
    assert sources == ["api.cu", "serve.cu"] and links == 1 and sum("-DOTHER" in c for c in calls) == 2
    tree.touch("pkg/csrc/serve.cu")
    assert tree.build()[0] == ["serve.cu"]


def test_the_library_needs_no_torch(tree):
    tree.monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None)
    assert tree.build()[:3] == (["api.cu", "serve.cu"], 1, 0)
    assert not tree.mod.needs_build() and tree.build(force=True)[:3] == (["api.cu", "serve.cu"], 1, 0)


def test_a_copied_tree_compiles_its_own_sources(tree, tmp_path):
    """Objects that were copied with the tree say nothing of the copy's sources."""
    tree.build()
    copy = tmp_path / "copy"
    shutil.copytree(tree.root / "pkg", copy / "pkg")
    shutil.copytree(tree.root / "include", copy / "include")
    spec = importlib.util.spec_from_file_location("_build_of_the_copy", copy / "pkg" / "build.py")
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert not mod.needs_library()
    (copy / "pkg" / "csrc" / "serve.cu").write_text("// changed")
    mod.build()
    assert "serve.cu" in tree.ran()[0]
