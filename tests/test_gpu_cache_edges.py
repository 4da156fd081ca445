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


# ------------------------------------------------------------------------------------------------------------------- preferences that mask
LOWEST = float(np.finfo(np.float32).min)


def check_masked(s):
    """The bound of Step.check with S, the scores' magnitude, taken over the keys that have weight and are not masked: masked scores that
    tie differ by nothing, in fp32 as in fp64, and those below others by more than either can hold."""
    torch.cuda.synchronize()
    O = f64(s.O)
    alpha, rho = f64(s.alpha), f64(s.rho)
    for r in range(len(s.lens)):
        a, n = int(s.offsets[r]), s.new[r]
        want, _, A, S = orc.attend(f64(s.q[a:a + n]), f64(s.k[r]), f64(s.v[r]), s.lens[r] - n, s.mask, alpha, rho, s.pos[r], None, None)
        for i in range(n):
            for h in np.nonzero(s.mask)[0]:
                x = np.array([alpha[h, j] + rho[h, s.pos[r][i] - j] for j in range(s.lens[r] - n + i + 1)])
                x = x[(x - x.max() > -200) & (np.abs(x) < 1e6)]
                S[i, h] = np.abs(x).max(initial=0.0)
        rel = 2 * (s.D + 6) * S[..., None] * 2.0 ** -23 + 2.0 ** -20 + 2 * (s.lens[r] + 64) * 2.0 ** -23
        bf = s.O.dtype == torch.bfloat16
        tol = A * (rel + (2.0 ** -8 if bf else 2.0 ** -22)) + np.abs(want) * (2.0 ** -8 if bf else 2.0 ** -24)
        bad = ~(np.abs(O[a:a + n] - want) <= tol)
        assert not bad.any(), (r, np.argwhere(bad)[:5], O[a:a + n][bad][:5], want[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("low", [LOWEST, -3e38, -2.2e38, -1e38, -1e30, -1.1e30, -1.7e30, -2.9e30, -1e18, -1.3e18, 1e30, 1.3e30])
@pytest.mark.parametrize("D,g,new,out", [(64, 1, 1, "bf16"), (128, 8, 1, "fp32"), (96, 8, 3, "bf16"), (64, 8, 40, "bf16"), (96, 8, 9, "bf16"), (128, 8, 5, "bf16"),
                                         (128, 8, 40, "fp32")])
def test_rows_whose_keys_are_masked_by_low_preferences(low, D, g, new, out):
    """Key preferences at a value that masks (the lowest of the type, -1e30 and others): alone they are all alike, beside others they do not
    count, and where they come first they leave nothing behind."""
    s = Step([300 + new, 70 + new, new], [new] * 3, 8, g, D, 16, "page", range(8), out=out, seed=21)
    s.alpha[0, :] = low                                     # every key
    s.alpha[1, :100] = low                                  # padding in front
    s.alpha[2, 20:] = low                                   # only the first keys count
    s.alpha[3, :] = low
    s.alpha[3, 40] = 0.5                                    # one key counts
    s.alpha[4, ::2] = low
    s.rho[5, 12:] = low                                     # a window
    s.alpha[6, :50] = low                                   # two values that mask
    s.alpha[6, 50:] = low / 2
    s.rho[7, :] = low
    s.call(saf.Context(0))
    check_masked(s)


@pytest.mark.parametrize("D,g,new", [(64, 1, 1), (128, 8, 3), (64, 8, 40), (128, 8, 40)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_rows_whose_low_preferences_are_split_over_blocks(D, g, new, out):
    s = Step([5000 + new], [new], 8, g, D, 64, "page", range(8), out=out, seed=22)
    s.alpha[0, :] = LOWEST
    s.alpha[1, :4000] = LOWEST
    s.alpha[2, 1000:] = LOWEST
    s.alpha[3, :] = -1e30
    s.alpha[4, :4500] = -1.3e30
    s.alpha[5, 30:] = -1e30
    s.alpha[6, :2500] = LOWEST
    s.alpha[6, 2500:] = -2.5e38                             # (past the type's range in powers of two, both)
    s.rho[7, :] = -1.7e30
    s.call(saf.Context(0))
    check_masked(s)


@pytest.mark.parametrize("D,g,new", [(64, 1, 1), (128, 8, 3), (64, 8, 40), (96, 8, 40), (128, 8, 40)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_large_magnitude(D, g, new, out, sign):
    """Queries and keys whose products are exact and large: 2^40 times small whole numbers that tie.  The largest take all."""
    s = Step([150 + new, new], [new] * 2, 8, g, D, 16, "page", (), out=out, scale=0.125, seed=23)
    rng = np.random.default_rng(24)
    s.q.zero_()
    s.q[..., 0] = 2.0 ** 20
    for r in range(2):
        j = np.arange(s.lens[r])
        p, at = s.table[r][torch.from_numpy(j // 16).cuda()].long(), torch.from_numpy(j % 16).cuda()
        c = torch.from_numpy(sign * rng.integers(3, 8, (s.lens[r], 8 // g))).cuda()
        s.k[r].zero_()
        s.k[r][..., 0] = c * 2.0 ** 20
        s.kc[p, :, at] = s.k[r]
    s.call(saf.Context(0))
    torch.cuda.synchronize()
    for r in range(2):
        a, n = int(s.offsets[r]), new
        want, lse, A, _ = orc.attend(f64(s.q[a:a + n]), f64(s.k[r]), f64(s.v[r]), s.lens[r] - n, s.mask, f64(s.alpha), f64(s.rho), s.pos[r], None, 0.125)
        half = 2.0 ** -8 if out == "bf16" else 2.0 ** -22   # (equal weights: no rounding but in the sums and on the way out)
        assert (np.abs(f64(s.O[a:a + n]) - want) <= (2.0 ** -20 + 2 * (s.lens[r] + 64) * 2.0 ** -23) * A + half * np.abs(want)).all()
        assert (np.abs(f64(s.LSE[a:a + n]) - lse) <= np.abs(lse) * 2.0 ** -22).all()


@pytest.mark.parametrize("D,g,new,out", [(64, 1, 1, "fp32"), (96, 8, 3, "bf16"), (64, 8, 40, "bf16"), (128, 8, 40, "bf16")])
def test_rows_whose_preferences_are_all_minus_infinity(D, g, new, out):
    s = Step([300 + new, 70 + new], [new] * 2, 8, g, D, 16, "page", (0, 2, 5), out=out, seed=25)
    s.alpha[0, :] = float("-inf")
    s.alpha[2, :100] = float("-inf")
    s.alpha[5, :], s.rho[5, :] = LOWEST, LOWEST             # (their sum in fp32)
    s.call(saf.Context(0))
    torch.cuda.synchronize()
    total = 2 * new
    assert not s.O[:total, 0].any() and not s.O[:total, 5].any()
    for i, pos in enumerate(int(x) for p in s.pos for x in p):
        assert bool(s.O[i, 2].any()) == (pos >= 100)        # (that head's first key with weight)
    assert torch.isfinite(s.O).all() and not s.LSE[:total, [0, 2, 5]].any()


# ------------------------------------------------------------------------------------------------------------------- rows that are not computed
def check_first(s, many, known=None):
    """The first `many` rows of each request against the oracle over all of its keys (`known`: new tokens of which keys are seen)."""
    torch.cuda.synchronize()
    bf = s.O.dtype == torch.bfloat16
    for r in range(len(s.lens)):
        a, n = int(s.offsets[r]), s.new[r]
        m = min(many, n)
        ctx, z = s.lens[r] - n, min(n, known or n)
        sets = [x & ((1 << z) - 1) for x in s.sets[r][:z]] if s.tree else None
        want, lse, A, S = orc.attend(f64(s.q[a:a + z]), f64(s.k[r][:ctx + z]), f64(s.v[r][:ctx + z]), ctx, s.mask, f64(s.alpha), f64(s.rho), s.pos[r][:z], sets, None)
        rel = 2 * (s.D + 6) * S[..., None] * 2.0 ** -23 + 2.0 ** -20 + 2 * (s.lens[r] + 64) * 2.0 ** -23
        tol = A * (rel + (2.0 ** -8 if bf else 2.0 ** -22)) + np.abs(want) * (2.0 ** -8 if bf else 2.0 ** -24)
        bad = ~(np.abs(f64(s.O[a:a + z]) - want) <= tol)[:m]
        assert not bad.any(), (r, np.argwhere(bad)[:5])
        fin = np.isfinite(lse[:m])
        assert np.array_equal(f64(s.LSE[a:a + m])[~fin], lse[:m][~fin])
        assert (np.abs(f64(s.LSE[a:a + m]) - np.where(fin, lse[:m], 0)) <= (rel[..., 0] + np.abs(lse) * 2.0 ** -22)[:m])[fin].all()
        assert (s.O[a + m:a + n] == 9.0).all() and (s.LSE[a + m:a + n] == 9.0).all()


@pytest.mark.parametrize("D,g,max_new,out", [(64, 2, 2, "bf16"), (128, 4, 3, "fp32"), (64, 4, 33, "bf16"), (96, 2, 34, "bf16"), (128, 2, 20, "bf16")])
@pytest.mark.parametrize("tree,positions", [(False, True), (False, False), (True, True)])
def test_rows_of_requests_that_bring_more_than_the_bound(D, g, max_new, out, tree, positions):
    """Rows up to the bound see what they see without it: the context, and of the new tokens their own."""
    new = [max_new + 4, 50, max_new, max_new + 1, 2]
    lens = [300 + new[0], 50, 64 + max_new, 17 + new[3], 90]
    s = Step(lens, new, 2 * g, g, D, 16, "page", (0,), out=out, tree=tree, positions=positions, max_new=max_new, seed=31)
    if tree:
        rng = np.random.default_rng(32)                     # later tokens in the sets, those behind the bound too
        s.sets = [[int(x) for x in rng.integers(0, 2 ** 63, n, dtype=np.uint64) & np.uint64((1 << n) - 1)] for n in new]
        s.masks = torch.from_numpy(np.array([x for t in s.sets for x in t] + [0] * 2, dtype=np.uint64).view(np.int64)).cuda()
    s.call(saf.Context(0))
    check_first(s, max_new)


@pytest.mark.parametrize("D,g,max_new", [(64, 2, 8), (128, 2, 64)])
def test_rows_of_a_prompt_longer_than_a_set(D, g, max_new):
    new = [200, 70, 65]
    s = Step([200, 300 + 70, 1 + 65], new, 2 * g, g, D, 16, "page", (0,), max_new=max_new, seed=33)
    s.call(saf.Context(0))
    check_first(s, max_new)


@pytest.mark.parametrize("D,g,new", [(64, 2, 6), (128, 4, 40)])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_of_a_request_that_ends_behind_the_last_row(D, g, new, tree):
    """Offsets past N: the rows that there are see their context and the new tokens that have rows."""
    s = Step([100 + new, 77 + new], [new, new], 2 * g, g, D, 16, "page", (0,), tree=tree, pad=0, seed=34)
    if tree:
        s.sets[1] = [(1 << new) - 1] * new
        s.masks = torch.from_numpy(np.array([x for t in s.sets for x in t], dtype=np.uint64).view(np.int64)).cuda()
    s.prob.N = new + 5
    s.call(saf.Context(0))
    torch.cuda.synchronize()
    assert (s.O[new + 5:] == 9.0).all() and (s.LSE[new + 5:] == 9.0).all()
    s.new, s.lens = [new, 5], [100 + new, 77 + 5]
    s.k[1], s.v[1], s.pos[1], s.sets[1] = s.k[1][:82], s.v[1][:82], s.pos[1][:5], [x & 31 for x in s.sets[1][:5]]
    check_first(s, new)


# ------------------------------------------------------------------------------------------------------------------- values that are not finite
@pytest.mark.parametrize("D,g,new", [(64, 1, 5), (96, 2, 7), (128, 4, 3), (64, 4, 40), (96, 2, 48), (128, 4, 40)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_cached_values_behind_a_frozen_rows_position_do_not_reach_it(D, g, new, what):
    ctx = 230
    s = Step([ctx + new, 90 + new], [new] * 2, 2 * g, g, D, 16, "page", (0, g), tree=True, seed=41)
    rng = np.random.default_rng(42)
    place(s, [rng.integers(40, ctx + new, new), s.pos[1]])
    context = saf.Context(0)
    s.call(context)
    s.check()
    clean, lse = s.O.clone(), s.LSE.clone()
    for hit in (45, 150, 229):                              # tiles of cached keys alone, and the one where the new tokens begin
        s.vc[int(s.table[0, hit // 16]), :, hit % 16, 3] = what
        s.call(context)
        torch.cuda.synchronize()
        for i in range(new):
            for h in range(2 * g):
                if s.mask[h] and s.pos[0][i] < hit:
                    assert torch.equal(s.O[i, h], clean[i, h]), (i, h, hit)
                else:
                    assert not torch.isfinite(s.O[i, h, 3]), (i, h, hit)
                    assert torch.isfinite(s.O[i, h, 4:]).all() and torch.isfinite(s.O[i, h, :3]).all()
        assert torch.equal(s.O[new:2 * new], clean[new:2 * new]) and torch.equal(s.LSE, lse)
        s.vc[int(s.table[0, hit // 16]), :, hit % 16, 3] = s.v[0][hit, :, 3]


# ------------------------------------------------------------------------------------------------------------------- waits that run out
# (the last of each pair: on 148 SMs block 1, or its first warp, holds the end of one unit and the beginning of the next)
@pytest.mark.parametrize("D,g,new,lens", [(64, 1, 1, [9000]), (64, 1, 1, [790, 9000]), (128, 4, 3, [5000, 3000]), (128, 4, 3, [270, 9000]),
                                          (64, 4, 33, [9000]), (64, 4, 33, [890, 890, 9000]), (128, 4, 40, [4000, 3000]), (128, 4, 33, [890, 890, 9000])])
def test_a_wait_that_runs_out_leaves_recorded_steps_whole(monkeypatch, D, g, new, lens):
    """The context's first attention call leaves out one copy of a tile (a host-side switch, off by default), so that waits reach their limit
    (20 ms here) in a block that holds parts of cut units.  The call is reported; a step recorded before the report is right."""
    monkeypatch.setenv("SAF_WAIT_LIMIT_MS", "20")
    monkeypatch.setenv("SAF_SELFTEST_DROP_LOAD", "1")
    ctx = saf.Context(0)
    monkeypatch.delenv("SAF_SELFTEST_DROP_LOAD")
    monkeypatch.delenv("SAF_WAIT_LIMIT_MS")
    s = Step(lens, [new] * len(lens), 2 * g, g, D, 16, "page", (0,), tree=True, seed=51)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.call(ctx)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        s.call(ctx)
    code, detail = ctx.saf_last_device_status()
    assert code == saf.SAF_ERR_DEVICE_TIMEOUT and (detail >> 24) & 0xFF == 1, (code, hex(detail))
    assert (detail >> 16) & 0xFF in (90, *range(111, 122)) and detail & 0xFFFF == 1, hex(detail)
    for _ in range(3):
        s.O.fill_(9.0), s.LSE.fill_(9.0), s.q.normal_(), s.vc.copy_(s.vc.roll(1, 3)), s.v.__setitem__(slice(None), [x.roll(1, 2) for x in s.v])
        torch.cuda.synchronize()
        graph.replay()
        s.check()
    assert ctx.saf_last_device_status()[0] == saf.SAF_OK
