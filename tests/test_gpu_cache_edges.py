"""Attention over the paged cache where a step departs from what a plan makes: positions that are not the tokens' places, preferences that
mask, more new tokens than are computed, values that are not finite, waits that run out.  Against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2609_34650_b200 as saf
from oracle import saf_cache_oracle as orc
from test_gpu_cache import Step, f64, ints

pytestmark = pytest.mark.gpu


def place(s, positions):
    """New tokens at these positions (a row of them for each request)."""
    s.pos = [np.asarray(p) for p in positions]
    s.positions = ints([int(x) for p in s.pos for x in p] + [-9] * (s.N - sum(s.new)))


# ------------------------------------------------------------------------------------------------------------------- positions
@pytest.mark.parametrize("shift", [1, 10, 40, 100])
@pytest.mark.parametrize("D,nf", [(64, 1), (64, 13), (96, 1), (96, 5), (128, 1), (128, 13)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_chains_ahead_of_their_places(D, nf, shift, out):
    """A prefix that the cache does not hold, as after evicted tokens: every position lies `shift` past the token's place."""
    new = [9, 32, 20, 9]
    lens = [1000 + 9, 64 + 32, 100 + 20, 9]
    s = Step(lens, new, 32, 16, D, 16, "page", tuple(range(nf)) + (20,), out=out, max_len=1200, seed=shift)
    place(s, [p + shift for p in s.pos])
    s.call_and_check()


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("tree", [False, True])
def test_row_tiles_of_one_request_at_positions_far_apart(D, out, tree):
    """The first tokens stand below the context, or far behind the others, whose own row tiles look like any chain's."""
    new = [40, 40, 40]
    s = Step([300 + 40, 130 + 40, 64 + 40], new, 32, 16, D, 16, "page", (0, 3, 20), out=out, tree=tree, max_len=700, seed=D)
    first, second, third = (p.copy() for p in s.pos)
    first[:16] = first[0] - 100 + np.arange(16)
    second[:16] = second[0] + 300 + np.arange(16)
    third[8:24] = np.arange(16) * 3
    place(s, [first, second, third])
    s.call_and_check()


@pytest.mark.parametrize("g,D,new", [(4, 64, 9), (4, 64, 40), (2, 96, 40), (1, 128, 9), (4, 128, 64)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_sets_with_later_tokens_and_no_positions(g, D, new, out):
    """Positions left out are the tokens' places, so a frozen row drops the later tokens of its set and an ordinary row sees them."""
    s = Step([200 + new, new, 65 + new], [new] * 3, 2 * g, g, D, 16, "page", (0, 2 * g - 1), out=out, tree=True, seed=new)
    rng = np.random.default_rng(new)
    s.sets = [[int(x) for x in rng.integers(0, 2 ** 63, new, dtype=np.uint64) & np.uint64((1 << new) - 1)] for _ in range(3)]
    s.masks = torch.from_numpy(np.array([x for t in s.sets for x in t] + [0] * 2, dtype=np.uint64).view(np.int64)).cuda()
    s.pos = [n - new + np.arange(new) for n in s.lens]
    s.positions = None
    s.call_and_check()
