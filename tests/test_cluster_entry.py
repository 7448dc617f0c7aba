"""Shared memory of another CTA may be reached only once that CTA is known to run: in every kernel that maps addresses of its
cluster's other CTAs, a barrier of the cluster comes first."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2101_01321_b200" / "csrc"
BARRIER = r"\bcluster_(?:sync|wait)\(\)"


def _bodies(text):
    """(name, body) of every function whose opening brace ends a line at the outer level of the file."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"^(?!namespace)[^\s#}/][^;{}]*?\b(\w+)\([^;{}]*\)\s*\{$", text, re.M):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), text[m.end():at]


SOURCES = sorted(p.name for p in CSRC.glob("*.cu") if "map_to_cta(" in p.read_text())


@pytest.mark.parametrize("source", SOURCES)
def test_a_barrier_of_the_cluster_comes_before_the_first_foreign_address(source):
    bodies = list(_bodies((CSRC / source).read_text()))
    first = BARRIER
    for name, body in bodies:                      # a helper that passes such a barrier counts where it is called
        if re.search(BARRIER, body) and "map_to_cta(" not in body and not name.endswith("_kernel"):
            first += rf"|\b{name}(?:<[^;()]*>)?\("
    users = [(name, body) for name, body in bodies if "map_to_cta(" in body]
    assert users, source
    for name, body in users:
        barrier = re.search(first, body)
        assert barrier and barrier.start() < body.index("map_to_cta("), (source, name)
