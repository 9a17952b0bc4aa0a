"""An issuing warp of the prompt kernel takes no tile of V before it has landed: the order of its waits, as it stands in the source, in a
model of the kernel's barriers with copies that complete in any order."""
import random
import re

import pytest

from prompt_waits import Early, Model, some_units, source


def weights_first():
    text = source()
    text = text[text.index("mma_16_ts(tO") - 3000:text.index("mma_16_ts(tO")]
    v, p = [m.start() for m in re.finditer(r"wait_warp\(v_full\(vst\)", text)], [m.start() for m in re.finditer(r"wait_warp\(p_full\(s, h\)", text)]
    assert len(v) == 1 and len(p) == 1
    return p[0] < v[0]


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
            Model(rng, some_units(rng), 2, False, True).run()
        except Early:
            early += 1
    assert early > 0
