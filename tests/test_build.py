"""Which objects the build takes for current, with a compiler that only writes files."""
import os
import subprocess
import sys

import pytest

from paper_2412_18052_b200 import build as b

COMPILER = '''#!{python}
import os, sys
args = sys.argv[1:]
source, out, listed = args[args.index("-c") + 1], args[args.index("-o") + 1], args[args.index("-MF") + 1]
header = os.path.join(os.path.dirname(source), "a.cuh")
with open(listed, "w") as f:
    f.write(out + " : " + source + " \\\\\\n")
    f.flush()
    if os.path.exists(os.path.join(os.path.dirname(source), "fail")):
        sys.exit(1)
    f.write("    " + header + "\\n")
open(out, "w").write("object")
'''


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A source and a header, both older than build.py, and a compiler."""
    compiler = tmp_path / "nvcc"
    compiler.write_text(COMPILER.format(python=sys.executable))
    compiler.chmod(0o755)
    monkeypatch.setenv("NVCC", str(compiler))
    for name in ("s.cu", "a.cuh"):
        (tmp_path / name).write_text("//")
        os.utime(tmp_path / name, (1e9, 1e9))
    monkeypatch.setattr(b, "OBJECTS", str(tmp_path / "objects"))
    monkeypatch.setattr(b, "SOURCES", [str(tmp_path / "s.cu")])
    return tmp_path


def test_an_object_is_current_until_something_that_went_into_it_changes(tree):
    source = b.SOURCES[0]
    assert not b._object_up_to_date(source)
    b._compile(False, False)
    assert b._object_up_to_date(source)
    assert sorted(os.listdir(b.OBJECTS)) == ["s.o", "s.o.d"]
    for name in ("s.cu", "a.cuh"):
        os.utime(tree / name)
        assert not b._object_up_to_date(source), name
        os.utime(tree / name, (1e9, 1e9))
        assert b._object_up_to_date(source)


def test_a_compilation_that_does_not_end_leaves_the_object_with_its_whole_list(tree):
    """Half a list beside the object of an earlier build would hide what changes from then on."""
    b._compile(False, False)
    (tree / "fail").write_text("")
    with pytest.raises(subprocess.CalledProcessError):
        b._compile(True, False)
    os.utime(tree / "a.cuh")
    assert not b._object_up_to_date(b.SOURCES[0])


def test_an_object_of_another_tree_is_not_taken(tree, monkeypatch):
    """A copied tree brings objects along, with lists of the first one's files: changes in the copy would not show."""
    b._compile(False, False)
    copy = tree / "copy"
    copy.mkdir()
    (copy / "s.cu").write_text("// changed")
    os.utime(copy / "s.cu", (1e9, 1e9))
    assert not b._object_up_to_date(str(copy / "s.cu"))


def test_other_flags_make_everything_anew(tree):
    """The flags stand in build.py: what is older than it is not current."""
    b._compile(False, False)
    then = os.path.getmtime(b.__file__) - 10
    os.utime(b._object_of(b.SOURCES[0]), (then, then))
    assert not b._object_up_to_date(b.SOURCES[0])
    lib = tree / "lib.so"
    lib.write_text("")
    os.utime(lib, (then, then))
    assert not b._up_to_date(str(lib))
