"""CPU-only checks of when the library is built again.  Nothing is compiled: a stand-in takes the compiler's place."""
import importlib.util
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Writes what nvcc would write: the object or the library, and the list of what was read, with paths as they were given.
STAND_IN = """#!{python}
import os, re, sys
a = sys.argv[1:]
open(a[a.index("-o") + 1], "w").write("made")
if "-c" in a:
    seen, todo = [], [a[a.index("-c") + 1]]
    while todo:
        f = todo.pop(0)
        if f not in seen:
            seen.append(f)
            todo += [os.path.join(os.path.dirname(f), n) for n in re.findall(r'#include "(.*?)"', open(f).read())]
    obj = a[a.index("-o") + 1]
    open(a[a.index("-MF") + 1], "w").write(obj + " : " + " \\\\\\n    ".join(seen[:1] + ["/usr/include/stdio.h"] + seen[1:]) + "\\n")
    open(os.environ["STAND_IN_LOG"], "a").write(os.path.basename(seen[0]) + "\\n")
"""


def _load(root):
    spec = importlib.util.spec_from_file_location("built_here", os.path.join(root, "paper_2502_06833_b200", "build.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Tree:
    """A checkout with this repository's sources, and its build script."""

    def __init__(self, root, log):
        self.root, self.log = root, log
        self.module = _load(root)

    def build(self):
        """Names of the sources that were compiled."""
        if os.path.exists(self.log):
            os.remove(self.log)
        self.module.build()
        return sorted(open(self.log).read().split()) if os.path.exists(self.log) else []

    def touch(self, path):
        path = os.path.join(self.root, path)
        assert os.path.exists(path)
        newest = max(os.path.getmtime(os.path.join(d, f)) for d, _, names in os.walk(self.root) for f in names)
        os.utime(path, (newest + 10, newest + 10))

    def settle(self):
        """Everything that is built counts as newer than every source."""
        built = os.path.join(self.root, "paper_2502_06833_b200", "build")
        newest = max(os.path.getmtime(os.path.join(d, f)) for d, _, names in os.walk(self.root) for f in names)
        for at, f in enumerate(sorted(os.listdir(built))):
            os.utime(os.path.join(built, f), (newest + 20, newest + 20))
        os.utime(os.path.join(self.root, "paper_2502_06833_b200", "libead_b200.so"), (newest + 30, newest + 30))


@pytest.fixture()
def tree(tmp_path, monkeypatch):
    def make(name, like=None):
        root = str(tmp_path / name)
        if like:
            shutil.copytree(like, root)                                  # keeps times, takes what was built along
        else:
            shutil.copytree(os.path.join(ROOT, "include"), os.path.join(root, "include"))
            os.makedirs(os.path.join(root, "paper_2502_06833_b200"))
            shutil.copytree(os.path.join(ROOT, "paper_2502_06833_b200", "csrc"), os.path.join(root, "paper_2502_06833_b200", "csrc"))
            shutil.copy2(os.path.join(ROOT, "paper_2502_06833_b200", "build.py"), os.path.join(root, "paper_2502_06833_b200"))
        return Tree(root, log)
    nvcc, log = tmp_path / "nvcc", str(tmp_path / "log")
    nvcc.write_text(STAND_IN.format(python=sys.executable))
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.setenv("STAND_IN_LOG", log)
    return make


ALL = ["ead_api.cu", "ead_decoder_api.cu", "ead_pass_api.cu"]
# what a change of a file builds again
CHANGES = [("paper_2502_06833_b200/csrc/rope_kernel.cuh", ["ead_pass_api.cu"]), ("paper_2502_06833_b200/csrc/ead_api.cu", ["ead_api.cu"]), ("include/ead.h", ALL),
           ("paper_2502_06833_b200/csrc/ptx_sm100.cuh", ALL), ("paper_2502_06833_b200/build.py", ALL)]


def test_first_build_and_nothing_to_do(tree):
    t = tree("here")
    assert t.build() == ALL
    t.settle()
    assert t.build() == []


@pytest.mark.parametrize("path,want", CHANGES)
def test_a_change_is_built(tree, path, want):
    t = tree("here")
    t.build()
    t.settle()
    t.touch(path)
    assert t.build() == want


@pytest.mark.parametrize("path,want", CHANGES)
def test_a_change_in_a_copied_tree_is_built(tree, path, want):
    """The objects came along from another place; the original's files do not count, and may be gone."""
    first = tree("here")
    first.build()
    first.settle()
    t = tree("there", like=first.root)
    shutil.rmtree(first.root)
    assert t.build() == []
    t.touch(path)
    assert t.build() == want


@pytest.mark.parametrize("known", ["", "garbage", "build/ead_pass_api.o : /elsewhere/csrc/ead_pass_api.cu /elsewhere/csrc/rope_kernel.cuh\n"])
@pytest.mark.parametrize("path", ["paper_2502_06833_b200/csrc/rope_kernel.cuh", "include/ead.h"])
def test_without_a_list_that_fits_every_header_counts(tree, known, path):
    """No list, one that says nothing, and one of absolute paths of another checkout."""
    t = tree("here")
    t.build()
    built = os.path.join(t.root, "paper_2502_06833_b200", "build")
    for f in os.listdir(built):
        if f.endswith(".d"):
            open(os.path.join(built, f), "w").write(known)
    t.settle()
    assert t.build() == []
    t.touch(path)
    assert t.build() == ALL


def test_a_header_that_is_gone_is_built_without(tree):
    t = tree("here")
    t.build()
    t.settle()
    extra = os.path.join(t.root, "paper_2502_06833_b200", "csrc", "extra.cuh")
    source = os.path.join(t.root, "paper_2502_06833_b200", "csrc", "ead_pass_api.cu")
    text = open(source).read()
    open(extra, "w").close()
    open(source, "w").write('#include "extra.cuh"\n' + text)
    t.touch("paper_2502_06833_b200/csrc/ead_pass_api.cu")
    assert t.build() == ["ead_pass_api.cu"]
    os.remove(extra)
    open(source, "w").write(text)
    t.settle()
    assert t.build() == ["ead_pass_api.cu"]                              # whatever its times say
    t.settle()
    assert t.build() == []
