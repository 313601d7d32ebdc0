"""CPU tests of what the build script knows about its parts: a header that is not among an object's dependencies would leave the
object as it was when the header changes, and link two layouts of one struct."""
import os
import re

import pytest

from paper_2008_04567_amd import build


def included(path, seen):
    """The repository's own files that `path` includes, directly or not."""
    with open(path) as f:
        names = re.findall(r'#\s*include\s+"([^"]+)"', f.read())
    for name in names:
        for at in (os.path.join(build.CSRC, name), os.path.join(build.INCLUDE, name)):
            if os.path.exists(at) and at not in seen:
                seen.add(at)
                included(at, seen)
    return seen


def parts(monkeypatch):
    """(object, its source, its dependencies) of a build of what is stale, none of which is run."""
    asked = []

    def stale(obj, deps):
        asked.append((obj, set(map(os.path.normpath, deps))))
        return True

    commands = []
    monkeypatch.setattr(build, "sources_newer_than_lib", lambda: True)
    monkeypatch.setattr(build, "_stale", stale)
    monkeypatch.setattr(build, "_run", lambda cmd: commands.append(cmd) or "")
    build.build_library(force=False)
    source = {cmd[cmd.index("-o") + 1]: cmd[cmd.index("-c") + 1] for cmd in commands if "-c" in cmd}
    return [(obj, source[obj], deps) for obj, deps in asked]


def test_every_included_file_is_a_dependency(monkeypatch):
    found = parts(monkeypatch)
    assert len(found) == 2 + build.N_PARTS + 3 + 1 + len(build.SEQUENCE_PARTS)
    for obj, source, deps in found:
        need = {os.path.normpath(p) for p in included(source, {source})}
        assert need <= deps, "%s: %s" % (os.path.basename(obj), sorted(os.path.basename(p) for p in need - deps))


@pytest.mark.parametrize("part", ["wpk_grouped", "wpk_linear_q8"])
def test_the_struct_that_two_parts_share_makes_both_stale(monkeypatch, part):
    deps = {os.path.basename(obj): deps for obj, _, deps in parts(monkeypatch)}[part + ".o"]
    assert os.path.normpath(os.path.join(build.CSRC, "wpk_grouped.h")) in deps
