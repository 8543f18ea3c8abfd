"""The order that the kernels over experts' rows and hidden states keep on the device, read from
their sources, and that the bounds-checked build covers them."""
import re

import pytest

from test_answers_order_cpu import functions


@pytest.mark.parametrize("name,count", [("experts.cu", 9), ("hidden.cu", 5)])
def test_kernels_wait_before_they_read_or_write(name, count):
    """Every kernel may begin while the one before it ends: it waits once, unconditionally, and before
    that touches shared memory alone."""
    bodies = [(n, b) for n, b in functions(name) if n.endswith("_kernel")]
    assert len(bodies) == count
    for n, b in bodies:
        assert b.count("pdl_wait();") == 1, n
        before = b[:b.index("pdl_wait();")]
        before = re.sub(r"(__shared__|extern)[^;]*;", "", before)
        assert not re.search(r"\b(A|W|J\.job|head|part|sums|x|rows|pos|tgt)\b\s*[\[.]", before), n
        for line in before.split(";"):
            assert not re.search(r"\breturn\b", line), n


def test_blocks_of_a_cluster_meet_before_they_end():
    """What a block reads of another's shared memory lies between two cluster barriers; the last is
    met by every thread."""
    bodies = dict(functions("experts.cu"))
    for n in ("expert_sort_kernel", "expert_scan_kernel"):
        b = bodies[n]
        first, last = b.index("load_peer("), b.rindex("load_peer(")
        assert "cluster_sync();" in b[:first] and "cluster_sync();" in b[last:], n
    b = dict(functions("hidden.cu"))["hidden_kernel"]
    assert b.index("cluster_sync();") < b.index("pair_commit(") < b.rindex("cluster_sync();")
    assert b.rindex("cluster_sync();") < b.index("pair_tmem_dealloc(")
    assert "bulk_wait();" in b[:b.rindex("cluster_sync();")]


def test_every_wait_of_the_products_is_bounded():
    for name in ("hidden.cu", "pair_mma.cuh"):
        for n, b in functions(name):
            assert "mbar_try_wait(" not in b and not re.search(r"while\s*\(", b), n
    assert "BOUTE_WAIT_NS" in dict(functions("pair_mma.cuh"))["pair_wait"]


@pytest.mark.parametrize("name,of", [
    ("experts.cu", ("expert", "row", "count_choices", "place_choices", "expert_count_kernel",
                    "expert_scan_kernel", "expert_place_kernel", "expert_combine_kernel",
                    "expert_combine_grad_kernel", "expert_shifted_grad_kernel",
                    "expert_query_grad_kernel")),
    ("hidden.cu", ("hidden_kernel", "hidden_join_kernel", "hidden_positions_kernel",
                   "hidden_dh_kernel", "hidden_align_kernel"))])
def test_functions_that_compute_indices_check_them(name, of):
    bodies = dict(functions(name))
    assert [f for f in of if "BOUTE_INB(" not in bodies[f]] == []
