"""The bounds-checked build covers the kernels over a model's answers: every unit that its report
names checks indices, and so does every function of theirs that computes one."""
import os
import re

import pytest

from paper_2602_10729_gb300 import build as bld
from test_answers_order_cpu import functions


def reported_units():
    with open(os.path.join(bld.CSRC, "abi.cu")) as f:
        return re.findall(r"bounds_read_(\w+)", f.read())


@pytest.mark.parametrize("unit", reported_units())
def test_every_unit_of_the_report_checks_indices(unit):
    with open(os.path.join(bld.CSRC, unit + ".cu")) as f:
        text = f.read()
    assert f"BOUTE_BOUNDS_READER({unit})" in text and "BOUTE_INB(" in text


@pytest.mark.parametrize("name,of", [
    ("logprobs.cu", ("load_whole", "store_piece", "token_logprobs_kernel",
                     "token_logprobs_grad_kernel")),
    ("scores.cu", ("part", "cluster_join", "answer_scores_kernel", "answer_scores_grad_kernel")),
    ("route.cu", ("load_words", "logit_at", "apply_groups", "keep_groups", "in_order",
                  "write_chosen", "route_pairs_kernel", "route_bound_kernel", "load", "clear_run",
                  "for_run", "route_grad_chosen_kernel", "route_grad_softmax_kernel"))])
def test_functions_that_compute_indices_check_them(name, of):
    bodies = dict(functions(name))
    assert [f for f in of if "BOUTE_INB(" not in bodies[f]] == []
