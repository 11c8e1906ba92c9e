"""The build keeps an object only while all that decides its content is as it was: source, headers, flags and compiler.  A stand-in
for the compiler writes down what it is called with (no GPU, no nvcc)."""
import os
import re

import pytest

from paper_2605_04711_b200 import build as M

COMPILER = r"""#!/bin/sh
if [ "$1" = --version ]; then echo "stand-in VERSION"; exit 0; fi
while [ $# -gt 0 ]; do
    case "$1" in -o) out="$2"; shift;; -c) src="$2"; shift;; esac
    shift
done
if [ -n "$src" ]; then echo "$src" >> LOG; cat "$src" > "$out"; else echo link >> LOG; echo linked > "$out"; fi
"""


class Tree:
    def __init__(self, tmp, monkeypatch):
        self.tmp, self.patch, self.log = tmp, monkeypatch, tmp / "log"
        for d in ("include", "csrc", "a", "b"):
            (tmp / d).mkdir()
        for name in ("one.cu", "two.cu", "three.cpp"):
            (tmp / "csrc" / name).write_text(name)
        (tmp / "csrc" / "common.cuh").write_text("common")
        for k, v in dict(HERE=str(tmp), ROOT=str(tmp), CSRC=str(tmp / "csrc"), LIB=str(tmp / "lib.so"), LIB_CHECKED=str(tmp / "lib_checked.so"),
                         SOURCES=["one.cu", "two.cu", "three.cpp"], HEADERS=[str(tmp / "csrc" / "common.cuh")]).items():
            monkeypatch.setattr(M, k, v)
        self.compiler("a", "1.0")

    def compiler(self, where, version):
        path = self.tmp / where / "nvcc"
        path.write_text(COMPILER.replace("LOG", str(self.log)).replace("VERSION", version))
        path.chmod(0o755)
        self.patch.setenv("NVCC", str(path))

    def built(self, touch="", **kw):
        """What a build compiles; touch: a source that is newer than the library from here on."""
        self.log.write_text("")
        if os.path.exists(M.LIB):                            # (the library itself is made whenever something is newer than it)
            os.utime(M.LIB, (1, 1))
        if os.path.exists(M.LIB_CHECKED):
            os.utime(M.LIB_CHECKED, (1, 1))
        if touch:
            (self.tmp / "csrc" / touch).write_text((self.tmp / "csrc" / touch).read_text() + "+")
        M.build(**kw)
        lines = self.log.read_text().split("\n")[:-1]
        assert lines[-1] == "link"
        return sorted(os.path.basename(s) for s in lines[:-1])


ALL = ["one.cu", "three.cpp", "two.cu"]


@pytest.fixture
def tree(tmp_path, monkeypatch):
    return Tree(tmp_path, monkeypatch)


def test_objects_follow_sources_and_headers(tree):
    assert tree.built() == ALL and tree.built() == []
    assert tree.built(touch="two.cu") == ["two.cu"] and tree.built() == []
    assert tree.built(touch="common.cuh") == ALL
    assert tree.built(force=True) == ALL


def test_objects_follow_the_compiler(tree):
    assert tree.built() == ALL
    tree.compiler("b", "1.0")                                # another path
    assert tree.built(touch="one.cu") == ALL
    tree.compiler("b", "1.1")                                # another version in the same place
    assert tree.built(touch="one.cu") == ALL and tree.built() == []


def test_objects_follow_the_flags(tree, monkeypatch):
    """The flags are those of build.py: an edited copy of it recompiles everything, and so does its library."""
    assert tree.built() == ALL
    source = open(M.__file__).read()
    other = re.sub(r'"-O3"', '"-O2"', source)
    assert other != source
    for k in ("HERE", "ROOT", "CSRC", "LIB", "LIB_CHECKED", "SOURCES", "HEADERS"):
        other += f"\n{k} = {getattr(M, k)!r}\n"
    path = tree.tmp / "build.py"
    path.write_text(other)
    scope = {"__name__": "build", "__file__": str(path)}
    exec(compile(other, str(path), "exec"), scope)
    assert scope["needs_build"](M.LIB)                       # (the file that holds the flags is newer than the library)
    tree.log.write_text("")
    scope["build"]()
    assert sorted(os.path.basename(s) for s in tree.log.read_text().split("\n")[:-2]) == ALL


def test_an_object_that_was_not_finished_is_made_again(tree):
    assert tree.built() == ALL
    good = os.environ["NVCC"]
    bad = tree.tmp / "b" / "nvcc"
    bad.write_text(open(good).read().replace('cat "$src" > "$out"', 'echo half > "$out"; exit 1'))
    bad.chmod(0o755)
    os.replace(bad, good)                                    # (the same path and version: only its outcome is another)
    with pytest.raises(Exception):
        tree.built(touch="one.cu")
    tree.compiler("a", "1.0")
    assert tree.built() == ["one.cu"]


def test_both_builds_keep_their_own_objects(tree):
    assert tree.built() == ALL and tree.built(checked=True) == ALL and tree.built() == [] and tree.built(checked=True) == []


def test_reports_of_the_compiler_do_not_change_an_object(tree):
    assert tree.built() == ALL and tree.built(verbose=True) == []
