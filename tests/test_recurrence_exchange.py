"""The exchange of the recurrence's maps over a cluster, read in the source: the memory model gives
no test that a wait of too narrow a scope would have to fail."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2108_06004_gb300", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def test_messages_are_acquired_at_the_scope_of_their_senders():
    """st.async of another CTA releases at the cluster's scope; a wait that acquires at its own CTA's
    does not synchronise with it."""
    common = source("recurrence.cuh")
    wait = re.search(r"template <bool CLUSTER>\s*__device__ __forceinline__ bool barrier_wait\(.*?\n}\n", common, re.S).group(0)
    cluster, own = re.search(r"if \(CLUSTER\)(.*?)else(.*)", wait, re.S).groups()
    assert "mbarrier.try_wait.parity.acquire.cluster.shared::cta" in cluster
    assert "mbarrier.try_wait.parity.acquire.cta.shared::cta" in own
    for name in ("k_recurrence.cu", "k_recurrence_back.cu"):
        waits = re.findall(r"barrier_wait(<\w+>)?\(&(\w+)[.](\w+)", source(name))
        assert {w for w in waits if w[1] == "table"} == {("<true>", "table", "arrived")}, name
        assert {w for w in waits if w[1] != "table"} == {("<false>", "sh", "full")}, name
