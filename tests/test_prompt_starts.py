"""Which sequences of token_start the prompt kernels take, by the kernels' own functions run on the host: none that starts below an
earlier entry, so no token is two sequences' and the work is never more than the host's check allows (a counter of 20 bits hands it out)."""
import os
import random
import subprocess

import pytest

import paper_2607_19456_b200 as moa
from paper_2607_19456_b200 import build as moa_build

HARNESS = r"""
#include <cstdio>
#include <vector>
#include "moa_prompt.cuh"
using namespace moa;
int main()
{
    int batch, tokens, g;
    while (scanf("%d %d %d", &batch, &tokens, &g) == 3) {
        std::vector<int32_t> starts(batch + 1);
        for (auto &x : starts) if (scanf("%d", &x) != 1) return 1;
        PromptArgs a = {};
        a.token_start = starts.data(); a.tokens = tokens; a.batch = batch; a.g = g; a.causal = 1;
        a.h_kv = 1; a.g_mul = (1u << 31) / g; a.g_sh = 31;      // (g a power of two)
        int floor = 0, bad, tiles, pieces;
        long long units = 0;
        for (int b = 0; b < batch; ++b) {
            const PromptSeq s = prompt_seq<false>(a, b, floor, bad);
            prompt_counts<false>(a, s, 128, 0x7fffffff, tiles, pieces);
            units += tiles;
            printf("%d %d %d ", s.first, s.n, bad != 0);
        }
        printf("%lld\n", units);
    }
}
"""


@pytest.fixture(scope="module")
def seen(tmp_path_factory):
    """What the functions make of lists of (batch, tokens, g, starts)."""
    folder = tmp_path_factory.mktemp("starts")
    (folder / "starts.cu").write_text(HARNESS)
    root = os.path.dirname(os.path.dirname(os.path.abspath(moa.__file__)))
    subprocess.run([moa_build.nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I" + os.path.join(root, "include"),
                    "-I" + moa_build.CSRC, "-o", str(folder / "starts"), str(folder / "starts.cu")], check=True)

    def run(cases):
        text = "\n".join("%d %d %d %s" % (len(st) - 1, tokens, g, " ".join(map(str, st))) for tokens, g, st in cases)
        lines = subprocess.run([str(folder / "starts")], input=text, capture_output=True, text=True, check=True).stdout.strip().split("\n")
        return [[int(x) for x in line.split()] for line in lines]

    return run


def taken(tokens, starts):
    """The rule, in so many words."""
    out = []
    for b in range(len(starts) - 1):
        first, end = starts[b], starts[b + 1]
        inside = [x for x in starts[:b] if 0 <= x <= tokens]
        out.append(0 <= first <= end <= tokens and first >= max(inside, default=0))
    return out


def test_no_token_is_two_sequences(seen):
    rng = random.Random(5)
    cases = [(256, 2, [0, 200, 100, 256]), (1 << 20, 1, [0, 1 << 20] * 2048 + [0]), (100, 8, [0, 50, 190, 100, 100]), (100, 1, [-5, 7, 9, -1, 9, 100]),
             (100, 1, [0, 2 ** 31 - 1, 5, 60, -2 ** 31, 60, 100])]
    for _ in range(300):
        tokens, n = rng.randrange(1, 2000), rng.randrange(1, 40)
        starts = sorted(rng.randrange(0, tokens + 1) for _ in range(n + 1))
        for _ in range(rng.randrange(0, 4)):
            starts[rng.randrange(n + 1)] = rng.choice([-3, 0, tokens, tokens + 1, rng.randrange(0, tokens + 1)])
        cases.append((tokens, rng.choice([1, 2, 8]), starts))
    for (tokens, g, starts), got in zip(cases, seen(cases)):
        batch, at, want = len(starts) - 1, 0, taken(tokens, starts)
        for b in range(batch):
            first, n, bad = got[3 * b:3 * b + 3]
            assert bad == (not want[b])
            assert n == (starts[b + 1] - starts[b] if want[b] else 0)
            if n:
                assert at <= first and first + n <= tokens
                at = first + n
        assert got[-1] <= -(-tokens * g // 128) + batch    # what the host's check of the capacity counts on
