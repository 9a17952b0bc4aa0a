"""An issuing warp of the prompt kernel takes no tile of V before it has landed: the order of its waits, as it stands in the source, in a
model of the kernel's barriers with copies that complete in any order."""
import random
import re

import pytest

from prompt_waits import Early, Model, some_units, source


def weights_first():
    """Of a step's number: whether the weights are waited for before V."""
    text = source()
    text = " ".join(text[:text.index("mma_16_ts(tO")].split()[-150:])
    late = re.search(r"const bool late = (u == \d+|true|false);", text)
    assert late and re.search(r"if \(h == 0\) ok = wait_warp\(late \? p_bar : v_bar, late \? p_par : v_par, abort_flag[^)]*\); "
                              r"ok = ok && wait_warp\(late \? v_bar : p_bar, late \? v_par : p_par, abort_flag[^)]*\); if \(!ok\) break;", text)
    assert len(re.findall(r"wait_warp\(", text)) == 2
    return {"true": lambda u: True, "false": lambda u: False}.get(late[1], lambda u: u == int(late[1].split()[-1]))


@pytest.mark.parametrize("stages", [2, 4])
def test_no_tile_is_used_before_it_has_landed(stages):
    order = weights_first()
    for seed in range(600):
        rng = random.Random(seed)
        Model(rng, some_units(rng), stages, order, True).run()


def test_the_model_sees_the_wrong_order():
    early = 0
    for seed in range(600):
        rng = random.Random(seed)
        try:
            Model(rng, some_units(rng), 2, lambda u: False, True).run()
        except Early:
            early += 1
    assert early > 0
