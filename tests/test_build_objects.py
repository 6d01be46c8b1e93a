"""When a translation unit is compiled again. The compiler is a stand-in that writes the files a real one would."""
import os
import shutil

import pytest

from paper_2412_16187_b200 import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A source, a header that it reads, and a compiler that notes what it is called for."""
    source, header, runs = tmp_path / "unit.cu", tmp_path / "part.cuh", []
    for p in (source, header):
        p.write_text("")
        os.utime(p, (1000, 1000))

    def compiler(cmd, check):
        out, deps = cmd[cmd.index("-o") + 1], cmd[cmd.index("-MF") + 1]
        old = build._OBJ_DIR + "/unit.d"
        runs.append(open(old).read() if os.path.exists(old) else None)  # what others find while this runs
        with open(deps, "w") as f:
            f.write("object: " + cmd[-1] + " \\\n  " + os.path.join(os.path.dirname(cmd[-1]), "part.cuh") + "\n")
        with open(out, "w") as f:
            f.write("x")

    monkeypatch.setattr(build, "_OBJ_DIR", str(tmp_path / "build"))
    monkeypatch.setattr(build.subprocess, "run", compiler)
    return source, header, runs


def test_an_object_is_kept_until_something_that_it_read_is_newer(tree):
    source, header, runs = tree
    for expected in (1, 1):
        obj = build._object(str(source), False, False, False)
        assert len(runs) == expected and os.path.exists(obj)
    os.utime(header, (1e11, 1e11))
    build._object(str(source), False, False, False)
    assert len(runs) == 2
    assert sorted(os.listdir(build._OBJ_DIR)) == ["unit.d", "unit.o"]  # nothing else is left behind


def test_the_list_of_what_was_read_is_whole_while_another_compiles(tree):
    source, header, runs = tree
    build._object(str(source), False, False, False)
    os.utime(header, (1e11, 1e11))
    build._object(str(source), False, False, False)
    assert runs[0] is None and "part.cuh" in runs[1]
    with open(build._OBJ_DIR + "/unit.d", "w") as f:  # cut off by a build that was killed
        f.write("obj")
    build._object(str(source), False, False, False)
    assert len(runs) == 3


def test_objects_of_a_copied_tree_are_not_taken_for_its_own(tree, monkeypatch):
    source, header, runs = tree
    build._object(str(source), False, False, False)
    other = source.parent / "copy"
    other.mkdir()
    for p in (source, header):
        shutil.copy2(p, other)
    shutil.copytree(build._OBJ_DIR, other / "build")
    monkeypatch.setattr(build, "_OBJ_DIR", str(other / "build"))
    (other / "part.cuh").write_text("changed")
    os.utime(other / "part.cuh", (1e11, 1e11))
    build._object(str(other / "unit.cu"), False, False, False)
    assert len(runs) == 2
