"""Blocks of a cluster reach each other's shared memory only once all of them have started: in the kernels' text, a
cluster barrier comes before the first address in another block's shared memory (no GPU needed)."""

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14672_gb300", "csrc")


def kernels():
    """(name, text from its name to the next kernel) of every kernel."""
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for part in re.split(r"\b__global__\b", text)[1:]:
            found.append((re.search(r"\b(k_\w+)\s*\(", part).group(1), part))
    return found


REMOTE = [(name, text) for name, text in kernels() if "mapa_rank(" in text]


def test_the_kernels_of_clusters_are_found():
    assert {name for name, _ in REMOTE} >= {"k_top_logits", "k_distill", "k_mx4_tc", "k_mx4_pair"}


@pytest.mark.parametrize("name,text", REMOTE, ids=[name for name, _ in REMOTE])
def test_a_barrier_before_the_first_remote_address(name, text):
    before = text[:text.index("mapa_rank(")]
    assert "cluster_sync()" in before or ("cluster_arrive()" in before and "cluster_wait()" in before)
    # an arrival comes before its wait
    assert "cluster_wait()" not in before or before.index("cluster_arrive()") < before.index("cluster_wait()")
