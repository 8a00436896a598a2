"""Builds libmmv.so (the C-ABI CUDA library, nvcc for sm_100a) and _serve.so (its binding to torch tensors) in-tree."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libmmv.so"
OBJ = PKG / "build"
SOURCES = [CSRC / "api.cu", CSRC / "serve.cu"]
BINDING = PKG / "_serve.so"
BINDING_SOURCE = CSRC / "torch_binding.cpp"
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


HEADERS = PKG.parent / "include"


def newer(deps, than: Path) -> bool:
    t = than.stat().st_mtime
    return any(d.stat().st_mtime > t for d in deps)


def needs_library() -> bool:
    return not LIB.exists() or newer([*CSRC.glob("*.cu"), *CSRC.glob("*.cuh"), *CSRC.glob("*.h"), *HEADERS.glob("*.h")], LIB)


def torch_dir() -> Path | None:
    spec = importlib.util.find_spec("torch")
    return Path(spec.origin).parent if spec else None


def binding_made_for() -> str:
    """What the extension is compiled against, besides its sources."""
    return f"{sys.implementation.cache_tag}\n{(torch_dir() / 'version.py').read_text()}"


def needs_binding() -> bool:
    if torch_dir() is None:                         # (nothing to bind to: the C library alone)
        return False
    made = OBJ / "binding"
    if not BINDING.exists() or not made.exists() or newer([BINDING_SOURCE, *HEADERS.glob("*.h")], BINDING):
        return True
    return made.read_text() != binding_made_for()


def needs_build() -> bool:
    return needs_library() or needs_binding()


def stale(source: Path, obj: Path, deps: Path, made: Path, command: str) -> bool:
    """Whether an object is older than its source or a file that it included when it was last compiled, or was compiled otherwise or elsewhere."""
    if not obj.exists() or not deps.exists() or not made.exists() or made.read_text() != command:
        return True
    names = deps.read_text().replace("\\\n", " ").partition(":")[2].split()
    t = obj.stat().st_mtime
    return str(source) not in names or any(not Path(n).exists() or Path(n).stat().st_mtime > t for n in names if not n.startswith("/usr/"))


def build(force: bool = False, verbose: bool = False) -> Path:
    if force or needs_library():
        build_library(force, verbose)
    if torch_dir() is not None and (force or needs_binding()):
        build_binding()
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> Path:
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-DNDEBUG"]
    flags += os.environ.get("MMV_NVCC_FLAGS", "").split()
    # one object per source, so that an edit recompiles (side by side) only the sources that include the edited file
    command = " ".join([NVCC, *flags])
    objs = [(s, *(OBJ / f"{s.stem}.{end}" for end in ("o", "d", "flags"))) for s in SOURCES]
    OBJ.mkdir(exist_ok=True)
    part = f".{os.getpid()}.tmp"
    running = [(subprocess.Popen([NVCC, *flags, *(["-Xptxas", "-v"] if verbose else []), "-MD", "-MF", f"{d}{part}", "-c", "-o", f"{o}{part}", str(s)]), o, d, made)
               for s, o, d, made in objs if force or stale(s, o, d, made, command)]
    if any([p.wait() for p, *_ in running]):
        raise RuntimeError("nvcc failed")
    for _, o, d, made in running:
        made.unlink(missing_ok=True)
        os.replace(f"{o}{part}", o)
        os.replace(f"{d}{part}", d)
        made.write_text(command)
    tmp = LIB.with_suffix(f".{os.getpid()}.tmp")
    subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", str(tmp), *(str(o) for _, o, *_ in objs)], check=True)
    os.replace(tmp, LIB)
    return LIB


def build_binding() -> Path:
    """The extension is linked to libmmv.so beside it; torch's libraries are the ones that the process has loaded."""
    torch = torch_dir()
    cuda = Path(NVCC).resolve().parent.parent
    include = [torch / "include", torch / "include/torch/csrc/api/include", sysconfig.get_paths()["include"], cuda / "include"]
    tmp = BINDING.with_suffix(f".{os.getpid()}.tmp")
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-DNDEBUG", *(f"-I{i}" for i in include), "-o", str(tmp),
                    str(BINDING_SOURCE), f"-L{torch / 'lib'}", f"-L{PKG}", "-l:libmmv.so", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python",
                    "-Wl,-rpath,$ORIGIN"], check=True)
    os.replace(tmp, BINDING)
    OBJ.mkdir(exist_ok=True)
    (OBJ / "binding").write_text(binding_made_for())
    return BINDING


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
