"""Kernels whose CTAs reach into one another's shared memory, read as text (CPU): a CTA's shared memory may be touched by others once the whole
cluster has started and until it ends, so that a barrier of the cluster stands before a kernel's first such access and one behind
its last.  On a GPU a missing one shows rarely: the CTAs of a cluster start within a few hundred cycles."""
import re

import pytest

from test_ordering_host import functions, read, sources

REMOTE = re.compile(r"\bmap_shared_rank\(|\bin_cta\(|\bmapa\.")
BARRIER = re.compile(r"\bcluster\.sync\(\)|\bcluster_sync\(\)|\bcluster\.barrier_wait\(\)")
HELPERS = ("in_cta", "cluster_sync")


def in_order(text):
    """A barrier of the cluster before the first remote access, another behind the last one."""
    remote, barriers = [m.start() for m in REMOTE.finditer(text)], [m.start() for m in BARRIER.finditer(text)]
    return not remote or (any(b < remote[0] for b in barriers) and any(b > remote[-1] for b in barriers))


@pytest.mark.parametrize("name", sources())
def test_a_cluster_has_started_before_its_shared_memory_is_reached(name):
    for fn, text in functions(read(name)):
        assert fn in HELPERS or in_order(text), f"{name}: {fn}"


def test_barriers_in_two_parts_are_in_two_parts():
    """A wait that no arrival precedes would wait for ever."""
    for name in sources():
        for fn, text in functions(read(name)):
            arrivals, waits = ([m.start() for m in re.finditer(r"cluster\.barrier_%s\(\)" % w, text)] for w in ("arrive", "wait"))
            assert len(arrivals) == len(waits) and all(a < w for a, w in zip(arrivals, waits)), f"{name}: {fn}"


def test_the_check_sees_a_missing_barrier():
    body = "A; *cluster.map_shared_rank(&s[rank], threadIdx.x) = mine; B; pdl_trigger();"
    for first, last, ok in (("", "cluster.sync()", False), ("cluster.sync()", "", False), ("cluster.sync()", "cluster.sync()", True),
                            ("cluster.barrier_arrive()", "cluster.sync()", False), ("cluster.barrier_arrive(); cluster.barrier_wait()", "cluster.sync()", True)):
        assert in_order(body.replace("A", first).replace("B", last)) == ok
