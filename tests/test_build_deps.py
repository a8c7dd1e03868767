"""What build.py holds a source to depend on is what the source includes, directly or not."""
import os
import re

import pytest

from paper_2206_10620_b200 import build

GENERATED = {"core_gen.inc": "gen_core.py", "blockgemm_core.inc": "gen_blockgemm.py"}      # what they are made by


def included(path, seen):
    with open(path) as f:
        text = f.read()
    for name in re.findall(r'^\s*#\s*include\s+"([^"]+)"', text, re.M):
        if name in GENERATED:
            seen.add(GENERATED[name])
            continue
        at = next(p for p in (os.path.join(build._CSRC, name), os.path.join(build._INC, name)) if os.path.exists(p))
        if os.path.basename(at) not in seen:
            seen.add(os.path.basename(at))
            included(at, seen)
    return seen


@pytest.mark.parametrize("source", build._SOURCES)
def test_a_source_is_compiled_again_when_what_it_includes_changes(source):
    names = lambda paths: {os.path.basename(p) for p in paths}      # noqa: E731
    need = included(os.path.join(build._CSRC, source), set())
    assert need <= names(build._INCLUDES[source])
    assert need | {source} <= names(build._DEPS)
