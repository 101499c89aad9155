"""The build step's kept objects, with a stand-in for the compiler: what is linked belongs to one command and one compiler."""
import os
import stat
import subprocess
import threading

import pytest

from paper_2605_29843_b200 import build as harp_build

# "Compiles" to the text <source>:<flags>:<version>, "links" by joining those; fails for the source named in FAIL_ON, and
# notes how many of it run at once beside the objects of another build.
NVCC = """#!/bin/bash
[ "$1" = --version ] && { cat "$(dirname "$0")/version"; exit 0; }
out=""; src=""; timing=plain; compile=0; objects=()
while [ $# -gt 0 ]; do
  case "$1" in
    -o) out="$2"; shift;;
    -c) compile=1;;
    -DHARP_TM_TIMING) timing=timing;;
    *.cu) src="$(basename "$1")";;
    *.o) objects+=("$1");;
  esac
  shift
done
if [ $compile = 1 ]; then
  printf 'half of' > "$out"
  [ "$src" = "$FAIL_ON" ] && exit 1
  echo "$src" >> "$(dirname "$0")/compiled"
  sleep ${DELAY:-0}
  echo "$src:$timing:$(cat "$(dirname "$0")/version")" > "$out"
else
  printf 'half of' > "$out"
  [ "$FAIL_ON" = link ] && exit 1
  cat "${objects[@]}" > "$out"
fi
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    src = tmp_path / "csrc"
    src.mkdir()
    sources = [str(src / n) for n in ("a.cu", "b.cu", "c.cu")]
    header = str(src / "h.h")
    for p in [*sources, header]:
        open(p, "w").close()
        os.utime(p, (1000, 1000))
    nvcc = tmp_path / "nvcc"
    nvcc.write_text(NVCC)
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IXUSR)
    (tmp_path / "version").write_text("1")
    call = tmp_path / "call.so"
    call.write_text("")
    for name, value in dict(LIB=str(tmp_path / "lib.so"), OBJECTS=str(tmp_path / "_build"), CALL=str(call), sources=lambda: sources,
                            headers_of_sources=lambda: [header]).items():
        monkeypatch.setattr(harp_build, name, value)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.delenv("HARP_TM_TIMING", raising=False)
    monkeypatch.delenv("HARP_FAST_TIMING", raising=False)
    os.utime(call)
    return tmp_path


def linked(tree):
    return (tree / "lib.so").read_text().split()


def touch(tree, name):
    """A source newer than every object"""
    p = tree / "csrc" / name
    later = max(os.path.getmtime(f) for f in [*(tree / "_build").iterdir(), tree / "lib.so"]) + 1
    os.utime(p, (later, later))


def test_only_what_changed(tree):
    harp_build.build()
    assert linked(tree) == ["a.cu:plain:1", "b.cu:plain:1", "c.cu:plain:1"]
    (tree / "compiled").unlink()
    touch(tree, "b.cu")
    harp_build.build()
    assert (tree / "compiled").read_text().split() == ["b.cu"] and linked(tree) == ["a.cu:plain:1", "b.cu:plain:1", "c.cu:plain:1"]


def test_a_build_of_other_flags_that_failed(tree, monkeypatch):
    harp_build.build()
    touch(tree, "b.cu")
    monkeypatch.setenv("HARP_TM_TIMING", "1")
    monkeypatch.setenv("FAIL_ON", "b.cu")
    with pytest.raises(subprocess.CalledProcessError):
        harp_build.build()
    monkeypatch.delenv("HARP_TM_TIMING")
    monkeypatch.delenv("FAIL_ON")
    harp_build.build()
    assert linked(tree) == ["a.cu:plain:1", "b.cu:plain:1", "c.cu:plain:1"]


def test_a_compile_that_failed_leaves_no_object(tree, monkeypatch):
    monkeypatch.setenv("FAIL_ON", "b.cu")
    with pytest.raises(subprocess.CalledProcessError):
        harp_build.build()
    assert not (tree / "_build" / "b.cu.o").exists() and not (tree / "lib.so").exists()
    monkeypatch.delenv("FAIL_ON")
    harp_build.build()
    assert sorted(p.name for p in tree.iterdir()) == ["_build", "call.so", "compiled", "csrc", "lib.so", "nvcc", "version"]


def test_a_link_that_failed_leaves_nothing_beside_the_sources(tree, monkeypatch):
    monkeypatch.setenv("FAIL_ON", "link")
    with pytest.raises(subprocess.CalledProcessError):
        harp_build.build()
    assert not [p.name for p in tree.iterdir() if p.name.startswith("lib")]


def test_another_compiler_at_the_same_path(tree):
    harp_build.build()
    (tree / "version").write_text("2")
    touch(tree, "c.cu")
    harp_build.build()
    assert linked(tree) == ["a.cu:plain:2", "b.cu:plain:2", "c.cu:plain:2"]


def test_two_builds_at_once(tree, monkeypatch):
    """The second one waits, finds the library built, and compiles nothing."""
    monkeypatch.setenv("DELAY", "0.3")
    threads = [threading.Thread(target=harp_build.build) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert linked(tree) == ["a.cu:plain:1", "b.cu:plain:1", "c.cu:plain:1"]
    assert sorted((tree / "compiled").read_text().split()) == ["a.cu", "b.cu", "c.cu"]
