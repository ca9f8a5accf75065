"""Which of the routing calls need the context's workspace, and that the header says so: without a GPU, underneath a stand-in for the HIP runtime."""
import os
import re

import pytest

from paper_2510_25590_amd import binding as rg
import launch_recorder
from test_expert_calls import F32, NO_ROWS, combine, route, run, slots  # noqa: F401 (run: a fixture)


@pytest.mark.parametrize("tokens,k", [(1, 1), (2048, 1), (4096, 1), (128, 32)])
def test_sorts_that_one_launch_does_need_none(run, tokens, k):  # noqa: F811
    _, (code, launches, _, message) = run([NO_ROWS, slots(tokens=tokens, k=k, experts=1024)])
    assert code == rg.OK and len(launches) == 1, message


@pytest.mark.parametrize("tokens,k", [(4097, 1), (2049, 2), (1 << 19, 32)])
def test_longer_sorts_need_it(run, tokens, k):  # noqa: F811
    _, (code, launches, _, message) = run([NO_ROWS, slots(tokens=tokens, k=k, experts=4)])
    assert code == rg.ERR_WORKSPACE and "workspace" in message and not launches
    _, (code, launches, _, message) = run([F32, slots(tokens=tokens, k=k, experts=1024)])
    assert code == rg.OK and len(launches) == 2, message


def test_the_choice_and_the_weighted_sum_need_none(run):  # noqa: F811
    for command in (route(tokens=1 << 19, k=32), route(tokens=70000, experts=256, groups=8, top_groups=4, best=2, given=1), combine(tokens=1 << 19, k=32, cols=64)):
        _, (code, launches, _, message) = run([NO_ROWS, command])
        assert code == rg.OK and len(launches) == 1, message


def test_the_header_says_so():
    text = open(os.path.join(launch_recorder.ROOT, "include", "regione.h")).read()
    of_slots = re.search(r"\* regione_expert_slots: (.*?)\n \* regione_expert_combine: ", text, re.S).group(1)
    assert "4096" in of_slots and "workspace" in of_slots and "REGIONE_ERR_WORKSPACE" in of_slots
