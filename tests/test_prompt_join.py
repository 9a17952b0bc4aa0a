"""At the end of a unit of few rows the two slots of the prompt kernel tell each other their references and sums: neither writes the next
unit's before the other one has read the last one's, also where a unit leaves it no tile."""
import random
import re

import pytest

from prompt_waits import Early, Model, some_units, source


def join_waits():
    text = source()
    end = text.index("ml[s * 128 + row] =")
    text = text[text.rindex("o_full(s), no", 0, end):end]  # from the last product of the unit on
    return re.search(r"if \(unread\) \{\s*ok = wait_warp\(parted, \(nj - 1\) & 1, abort_flag[^)]*\);\s*unread = false;\s*if \(!ok\) break;", text) is not None


@pytest.mark.parametrize("stages", [2, 4])
def test_nothing_is_written_before_it_has_been_read(stages):
    order = join_waits()
    for seed in range(600):
        rng = random.Random(seed)
        Model(rng, some_units(rng), stages, lambda u: u == 0, order).run()


def test_the_model_sees_a_join_without_the_wait():
    early = 0
    for seed in range(200):
        rng = random.Random(seed)
        try:
            Model(rng, some_units(rng), 2, lambda u: u == 0, False).run()
        except Early:
            early += 1
    assert early > 0
