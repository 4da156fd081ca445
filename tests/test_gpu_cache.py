"""A step on a paged cache on the GPU against the fp64 oracle: plan, append, attention, and steps as they follow one another."""
import numpy as np
import pytest
import torch

import paper_2609_34650_b200 as saf
from oracle import saf_cache_oracle as orc

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------------------------- plan
class Pages:
    """Host mirror of a plan's state and its device arrays."""

    def __init__(self, R, N, page, n_pages, max_pages, seed=0, tree=False):
        self.R, self.N, self.page, self.n_pages, self.max_pages, self.tree = R, N, page, n_pages, max_pages, tree
        self.free = [int(x) for x in np.random.default_rng(seed).permutation(n_pages)]
        self.held, self.table = [0] * R, np.zeros((R, max_pages), np.int32)
        self.cache = saf.make_cache(R, N, page, n_pages, max_pages)
        self.d_held, self.d_count = ints(self.held), ints([n_pages])
        self.d_free, self.d_table = ints(self.free), torch.zeros((R, max_pages), dtype=torch.int32, device="cuda")
        self.out = {k: torch.full((n,), -77, dtype=torch.int32, device="cuda") for k, n in
                    (("offsets", R + 1), ("kv_lens", R), ("slots", N), ("positions", N), ("missing", R))}
        self.masks = torch.full((N,), -77, dtype=torch.int64, device="cuda") if tree else None

    def device(self, ctx, lens, new, parents, in_place=True):
        held, count = (self.d_held, self.d_count) if in_place else (torch.full_like(self.d_held, -5), torch.full_like(self.d_count, -5))
        ctx.saf_cache_plan(self.cache, lens, new, parents, self.d_held, held, self.d_count, count, self.d_free, self.d_table,
                           self.out["offsets"], self.out["kv_lens"], self.out["slots"], self.out["positions"], self.masks, self.out["missing"])
        self.d_held, self.d_count = held, count

    def step(self, ctx, lens, new, parents=None, in_place=True):
        self.device(ctx, ints(lens), ints(new), None if parents is None else ints(parents), in_place)
        want = orc.plan(lens, new, parents, self.held, self.free, self.table, self.page, self.max_pages, self.N)
        torch.cuda.synchronize()
        for k in ("offsets", "kv_lens", "slots", "positions", "missing"):
            assert np.array_equal(self.out[k].cpu().numpy(), np.array(want[k])), k
        assert self.d_held.tolist() == want["held"] and self.d_count.tolist() == [len(want["free"])]
        assert self.d_free.tolist()[:len(want["free"])] == want["free"]
        assert np.array_equal(self.d_table.cpu().numpy(), want["table"])
        if self.tree:
            assert np.array_equal(self.masks.cpu().numpy().view(np.uint64), want["masks"])
        self.held, self.free, self.table = want["held"], want["free"], want["table"]
        taken = [int(x) for r in range(self.R) for x in self.table[r, :self.held[r]]]
        assert sorted(taken + self.free) == list(range(self.n_pages))       # every page in one place
        return want


@pytest.mark.parametrize("R,page,n_pages,max_pages", [(1, 16, 8, 8), (7, 16, 60, 20), (33, 1, 400, 64), (600, 32, 3000, 9), (5, 48, 12, 6)])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("tree", [False, True])
def test_plan_over_many_steps(R, page, n_pages, max_pages, in_place, tree):
    rng = np.random.default_rng(R)
    ctx = saf.Context(0)
    N = max(70, R * 8)
    s = Pages(R, N, page, n_pages, max_pages, seed=1, tree=tree)
    lens = [0] * R
    for step in range(12):
        new = [int(x) for x in rng.integers(0, max(2, min(70, 2 * N // R)), R) * (rng.random(R) < 0.7)]
        lens = [0 if rng.random() < 0.15 else x for x in lens]              # some end, others begin
        if step == 5:
            lens[R // 2] = -1
        if step == 6:
            lens[R // 2], new[0] = 0, -3
        parents = [int(x) for x in rng.integers(-2, 66, N)] if tree and step % 3 == 2 else [int(rng.integers(-1, 1 + i % 40)) for i in range(N)] if tree else None
        want = s.step(ctx, lens, new, parents, in_place)
        # some drafted tokens are dropped
        lens = [max(0, k - int(rng.integers(0, 3))) if m == 0 else max(x, 0) for k, m, x in zip(want["kv_lens"], want["missing"], lens)]


def test_plan_of_the_largest_sizes():
    ctx = saf.Context(0)
    R, N = 4096, 9000
    s = Pages(R, N, 16, 40000, 12)
    rng = np.random.default_rng(0)
    for _ in range(3):
        s.step(ctx, [int(x) for x in rng.integers(0, 170, R)], [int(x) for x in rng.integers(0, 5, R)])


def test_plan_of_long_prompts():
    ctx = saf.Context(0)
    s = Pages(3, 100000, 16, 9000, 4096)
    s.step(ctx, [0, 0, 0], [33333, 1, 60000])
    s.step(ctx, [33333, 1, 60000], [1, 1, 0])


def test_plan_in_a_graph_serves_other_lengths():
    ctx = saf.Context(0)
    s = Pages(6, 64, 16, 100, 16, tree=True)
    lens, new, parents = ints([0] * 6), ints([3] * 6), ints([-1] * 64)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.device(ctx, lens, new, parents)
    rng = np.random.default_rng(3)
    host = [0] * 6
    for _ in range(4):
        n = [int(x) for x in rng.integers(0, 12, 6)]
        p = [int(rng.integers(-1, 1 + i % 9)) for i in range(64)]
        lens.copy_(ints(host)), new.copy_(ints(n)), parents.copy_(ints(p))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = orc.plan(host, n, p, s.held, s.free, s.table, 16, 16, 64)
        assert np.array_equal(s.out["slots"].cpu().numpy(), want["slots"]) and s.d_count.item() == len(want["free"])
        assert np.array_equal(s.masks.cpu().numpy().view(np.uint64), want["masks"])
        s.held, s.free, s.table = want["held"], want["free"], want["table"]
        host = want["kv_lens"]


def test_plan_refusals():
    ctx = saf.Context(0)

    def refused(change, drop=None, masks=True):
        s = Pages(4, 8, 16, 10, 5, tree=True)
        if change:
            setattr(s.cache, *change)
        a = [ints([1] * 4), ints([1] * 4), ints([-1] * 8), s.d_held, s.d_held, s.d_count, s.d_count, s.d_free, s.d_table, s.out["offsets"],
             s.out["kv_lens"], s.out["slots"], s.out["positions"], s.masks if masks else None, s.out["missing"]]
        if drop is not None:
            a[drop] = None
        with pytest.raises(saf.SafError) as e:
            ctx.saf_cache_plan(s.cache, *a)
        assert e.value.code == 1

    for change in (("R", 0), ("R", 4097), ("N", 0), ("page_size", 0), ("n_pages", 0), ("max_pages", 0), ("n_pages", 1 << 28), ("max_pages", 1 << 30)):
        refused(change)
    for i in range(15):
        refused(None, drop=i)


# ------------------------------------------------------------------------------------------------------------------- append
def pool(pages, heads, page, D, layout, fill=None, gen=None):
    shape = (pages, page, heads, D) if layout == "slot" else (pages, heads, page, D)
    t = torch.randn(shape, generator=gen, device="cuda").bfloat16() if fill is None else torch.full(shape, fill, device="cuda", dtype=torch.bfloat16)
    return t.transpose(1, 2) if layout == "slot" else t


@pytest.mark.parametrize("layout", ["page", "slot"])
@pytest.mark.parametrize("Hq,Hk,D,rot,inter,page", [(12, 12, 64, 64, False, 16), (8, 2, 128, 96, True, 16), (4, 4, 96, 96, False, 64), (6, 3, 64, 0, False, 1), (0, 2, 96, 20, True, 48),
                                                    (3, 1, 40, 40, False, 5)])
@pytest.mark.parametrize("N", [1, 7, 3000])
def test_append(layout, Hq, Hk, D, rot, inter, page, N):
    gen = torch.Generator(device="cuda").manual_seed(1)
    ctx = saf.Context(0)
    pages = (N + 40) // page + 3
    qkv = torch.randn((N, Hq + 2 * Hk, D), generator=gen, device="cuda").bfloat16()
    q, k, v = qkv[:, :Hq] if Hq else None, qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    kc, vc = pool(pages, Hk, page, D, layout, gen=gen), pool(pages, Hk, page, D, layout, gen=gen)
    before = kc.clone(), vc.clone()
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:N].int()
    gone = torch.rand(N, generator=gen, device="cuda") < 0.2
    slots = torch.where(gone, torch.where(torch.arange(N, device="cuda") % 2 == 0, -1, pages * page), slots).int().contiguous()
    pos = torch.randint(0, 100000, (N,), generator=gen, device="cuda").int()
    freqs = saf.saf_rotary_freqs(rot)[0] if rot else np.zeros(0)
    f = torch.from_numpy(freqs).cuda() if rot else None
    qo = torch.full((N, Hq, D), 7.0, device="cuda", dtype=torch.bfloat16) if Hq else None
    c = saf.make_cache(4, N, page, pages, 8, k_cache=kc, v_cache=vc, v_like=v)
    ctx.saf_cache_append(c, saf.make_rotary(q, k, qo, None, rot, inter), q, k, v, slots, pos if rot else None, f, qo, kc, vc)
    torch.cuda.synchronize()
    where = pos.cpu().numpy()[None]
    tol = lambda x, want: 2 * 8 * 2.0 ** -23 * np.abs(x).max() + 2.0 ** -8 * np.abs(want)  # noqa: E731
    turn = lambda t: orc.rotary(f64(t).transpose(1, 0, 2)[None], where, freqs, inter)[0].transpose(1, 0, 2)  # noqa: E731
    keep = ~gone.cpu().numpy()
    if Hq:
        want = turn(q)
        assert (np.abs(f64(qo) - want) <= tol(f64(q), want))[keep].all()
        assert (f64(qo)[~keep] == 7.0).all()
    wk, wv = f64(before[0]), f64(before[1])
    touched = np.zeros((pages, page), bool)
    at = slots.cpu().numpy()[keep]
    touched[at // page, at % page] = True
    new_k = turn(k)[keep]
    got = f64(kc)[at // page, :, at % page]
    assert (np.abs(got - new_k) <= tol(f64(k), new_k)).all()
    wv[at // page, :, at % page] = f64(v)[keep]
    assert np.array_equal(f64(vc), wv)
    assert np.array_equal(f64(kc).transpose(0, 2, 1, 3)[~touched], wk.transpose(0, 2, 1, 3)[~touched])


def test_append_refusals():
    ctx = saf.Context(0)
    N, H, D, page, pages = 4, 2, 64, 16, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((N, H, D), generator=gen, device="cuda").bfloat16() for _ in range(3))
    kc, vc = pool(pages, H, page, D, "page", 0.0), pool(pages, H, page, D, "page", 0.0)
    qo = torch.zeros_like(q)
    slots, pos = ints([0, 1, 2, 3]), ints([0, 1, 2, 3])
    f = torch.from_numpy(saf.saf_rotary_freqs(64)[0]).cuda()

    def refused(code, change_c=None, change_r=None, **args):
        c = saf.make_cache(2, N, page, pages, 8, k_cache=kc, v_cache=vc, v_like=v)
        r = saf.make_rotary(q, k, qo, None, 64)
        if change_c:
            setattr(c, *change_c)
        if change_r:
            setattr(r, *change_r)
        a = {"q": q, "k": k, "v": v, "slots": slots, "pos": pos, "f": f, "qo": qo, "kc": kc, "vc": vc, **args}
        with pytest.raises(saf.SafError) as e:
            ctx.saf_cache_append(c, r, *(a[n] for n in ("q", "k", "v", "slots", "pos", "f", "qo", "kc", "vc")))
        assert e.value.code == code

    for change in (("N", 5), ("H", 3), ("H", 0), ("D", 128), ("page_size", 0), ("kv_group", 3), ("kv_group", -1), ("n_pages", 0)):
        refused(1, change_c=change)
    for change in (("B", 2), ("T", 3), ("Hk", 1), ("D", 96), ("rot_dim", 80)):
        refused(1, change_r=change)
    for change in (("in_dtype", 1), ("out_dtype", 1)):
        refused(2, change_r=change)
    for name in ("q", "k", "v", "slots", "pos", "f", "qo", "kc", "vc"):
        refused(1, **{name: None})
    for name, t in (("q", q), ("k", k), ("v", v), ("qo", qo), ("kc", kc), ("vc", vc)):
        refused(1, **{name: t.flatten()[1:]})
    torch.cuda.synchronize()
    assert not kc.any() and not vc.any() and not qo.any()


# ------------------------------------------------------------------------------------------------------------------- attention
class Step:
    """A step over given lengths: pools with pages anywhere, rows packed, slots that hold nothing poisoned."""

    def __init__(self, lens, new, H, g, D, page=16, layout="page", frozen=(), tree=False, out="bf16", positions=True, max_new=None, max_len=None,
                 seed=0, pad=2, poison=float("nan"), scale=0.0, sliced=False, spare=3):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.new, self.H, self.g, self.D, self.scale = lens, new, H, g, D, scale
        R, Hk = len(lens), H // g
        self.N = sum(new) + pad
        self.max_new = max_new or max(new + [1])
        self.max_len = max_len or max(lens + [1])
        max_pages = -(-max(self.max_len, max(lens)) // page) + 1
        need = [-(-n // page) for n in lens]
        pages = sum(need) + spare
        ids = rng.permutation(pages)
        table = rng.integers(0, pages, (R, max_pages)).astype(np.int32)
        at = 0
        for r in range(R):
            table[r, :need[r]] = ids[at:at + need[r]]
            at += need[r]
        self.kc, self.vc = pool(pages, Hk, page, D, layout, poison), pool(pages, Hk, page, D, layout, poison)
        self.k, self.v = [], []
        for r in range(R):
            k, v = (torch.randn((lens[r], Hk, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
            j = np.arange(lens[r])
            p, s = torch.from_numpy(table[r][j // page].astype(np.int64)).cuda(), torch.from_numpy(j % page).cuda()
            self.kc[p, :, s], self.vc[p, :, s] = k, v
            self.k.append(k), self.v.append(v)
        wide = torch.randn((self.N, H + 2, D + 8), generator=gen, device="cuda").bfloat16()
        self.q = wide[:, 1:H + 1, 8:] if sliced else wide[:, :H, :D].contiguous()
        dt = torch.float32 if out == "fp32" else torch.bfloat16
        self.O = torch.full((self.N, H + 1, D + 8), 9.0, device="cuda", dtype=dt)[:, :H, :D] if sliced else torch.full((self.N, H, D), 9.0, device="cuda", dtype=dt)
        self.LSE = torch.full((self.N, H), 9.0, device="cuda")
        self.mask = np.zeros(H, np.uint8)
        self.mask[list(frozen)] = 1
        Tp = self.max_len + 5
        self.alpha = torch.randn((H, Tp), generator=gen, device="cuda")
        self.rho = -0.02 * torch.arange(Tp, device="cuda").float() + 0.1 * torch.randn((H, Tp), generator=gen, device="cuda")
        self.offsets = np.concatenate([[0], np.cumsum(new)])
        self.pos, self.sets = [], []
        for r in range(R):
            ctx = lens[r] - new[r]
            sets, depth = orc.ancestors([int(rng.integers(-1, i)) if i else -1 for i in range(new[r])])
            self.sets.append(sets)
            self.pos.append(ctx + (np.array(depth, int) if tree else np.arange(new[r])))
        self.tree = tree
        self.masks = None
        if tree:
            self.masks = torch.from_numpy(np.array([x for s in self.sets for x in s] + [0] * pad, dtype=np.uint64).view(np.int64)).cuda()
        self.positions = ints([int(x) for p in self.pos for x in p] + [-9] * pad) if positions or tree else None
        self.table, self.d_off, self.d_lens = torch.from_numpy(table).cuda(), ints(self.offsets.tolist()), ints(lens)
        self.prob = saf.make_cache(R, self.N, page, pages, max_pages, k_cache=self.kc, v_cache=self.vc, q_like=self.q, o_like=self.O, Tp=Tp,
                                   max_len=self.max_len, max_new=self.max_new, softmax_scale=scale)

    def call(self, ctx, lse=True):
        ctx.saf_cache_attn(self.prob, self.q, self.kc, self.vc, self.table, self.d_off, self.d_lens, self.positions, self.masks, self.mask,
                           self.alpha, self.rho, self.O, self.LSE if lse else None)

    def check(self, only=None):
        torch.cuda.synchronize()
        O, L = f64(self.O), f64(self.LSE)
        for r in range(len(self.lens)) if only is None else only:
            a, n = int(self.offsets[r]), self.new[r]
            if n == 0:
                continue
            want, lse, A, S = orc.attend(f64(self.q[a:a + n]), f64(self.k[r]), f64(self.v[r]), self.lens[r] - n, self.mask, f64(self.alpha), f64(self.rho),
                                         self.pos[r], self.sets[r] if self.tree else None, self.scale if self.scale > 0 else None)
            # A score is a sum of D exact products in fp32, each addition off by up to a step (2^-23) of the sum of their magnitudes S, then scaled
            # by log2(e) (or, frozen, a sum and a product of magnitude S): (D + 6) S 2^-23.  It moves a weight and the sum by that much each,
            # relatively; exponentials 2^-21; sums over the keys and over parts of them (len + 64) steps.  Weights may be rounded to bf16
            # where O is bf16 (half a step, 2^-8, of each), or to 24 bits; O is rounded to its type.
            rel = 2 * (self.D + 6) * S[..., None] * 2.0 ** -23 + 2.0 ** -20 + 2 * (self.lens[r] + 64) * 2.0 ** -23
            bf = self.O.dtype == torch.bfloat16
            tol = A * (rel + (2.0 ** -8 if bf else 2.0 ** -22)) + np.abs(want) * (2.0 ** -8 if bf else 2.0 ** -24)
            bad = ~(np.abs(O[a:a + n] - want) <= tol)
            assert not bad.any(), (r, np.argwhere(bad)[:5], O[a:a + n][bad][:5], want[bad][:5], tol[bad][:5])
            fin = np.isfinite(lse)
            assert np.array_equal(L[a:a + n][~fin], lse[~fin])
            assert (np.abs(L[a:a + n] - np.where(fin, lse, 0)) <= rel[..., 0] + np.abs(lse) * 2.0 ** -22)[fin].all()
        total = int(self.offsets[-1])
        assert (O[total:] == 9.0).all() and (L[total:] == 9.0).all()        # rows behind the last request
        return self


GEOMETRY = [(12, 1, 64, (1, 5, 7)), (16, 4, 64, (0, 3, 4, 5, 6, 7)), (6, 1, 96, (2,)), (8, 4, 128, (0, 6)), (16, 8, 128, ()), (4, 1, 128, (0, 1, 2, 3)), (6, 3, 96, (0, 1, 2))]


@pytest.mark.parametrize("layout,page", [("page", 16), ("slot", 48)])
@pytest.mark.parametrize("H,g,D,frozen", GEOMETRY)
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_one_token_a_request(H, g, D, frozen, layout, page, out):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 500, 1, 1031, 64]
    Step(lens, [1] * len(lens), H, g, D, page, layout, frozen, out=out).call_and_check()


@pytest.mark.parametrize("H,g,D,frozen", GEOMETRY)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("new", [[2, 5, 1, 0, 3, 8], [17, 32, 0, 33, 64, 1], [64, 63, 9, 40, 16, 31]])
def test_several_tokens_a_request(H, g, D, frozen, tree, new):
    lens = [n + c for n, c in zip(new, [0, 200, 15, 40, 777, 128])]
    Step(lens, new, H, g, D, 16, "page", frozen, tree=tree, seed=2).call_and_check()


@pytest.mark.parametrize("new,tree", [(1, False), (4, True), (40, True)])
@pytest.mark.parametrize("H,g,D,frozen", GEOMETRY[:4])
def test_long_contexts_are_split_and_joined(H, g, D, frozen, new, tree):
    lens = [9000, 5000 + new, 12345]
    Step(lens, [new] * 3, H, g, D, 64, "slot", frozen, tree=tree, out="fp32" if new == 4 else "bf16", seed=4).call_and_check()


def test_slices_positions_scale_and_no_lse():
    s = Step([70, 33], [3, 2], 8, 4, 64, 32, "slot", (1, 4), sliced=True, scale=0.07, positions=False)
    s.call_and_check()
    O = s.O.clone()
    s.O.fill_(9.0)
    s.call(saf.Context(0), lse=False)
    assert torch.equal(O, s.O)


def test_many_requests():
    lens = [1 + (i * 37) % 300 for i in range(700)]
    Step(lens, [1] * 700, 4, 2, 64, 16, "page", (1,), seed=5).call_and_check(only=range(0, 700, 23))


def test_idle_requests_and_rows_that_see_nothing():
    s = Step([5, 0, 40], [2, 0, 3], 4, 1, 64, frozen=(1,), tree=True)
    ctx = saf.Context(0)
    s.call(ctx)
    s.check()
    # the middle request's rows lie in a cache that the plan did not give it: length 0, two rows; and a tree row with no key at all
    s = Step([2, 40], [2, 3], 4, 1, 64, frozen=(1,), tree=True)
    s.d_lens[0] = 0
    s.call(ctx)
    s.check(only=[1])
    assert not s.O[:2].any() and torch.isinf(s.LSE[:2, [0, 2, 3]]).all() and (s.LSE[:2, [0, 2, 3]] < 0).all() and not s.LSE[:2, 1].any()
    s = Step([2, 40], [2, 3], 4, 1, 64, frozen=(1,), tree=True)
    s.masks[1] = 0
    s.call(ctx)
    s.check(only=[1])
    assert not s.O[1].any() and s.O[0].any()


@pytest.mark.parametrize("H,g,D,frozen", [(4, 1, 64, (1,)), (8, 4, 128, (2,)), (4, 2, 96, (0, 1))])
@pytest.mark.parametrize("new", [7, 40])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_does_not_reach_it(H, g, D, frozen, new, what):
    """NaN and infinities in a drafted token's key and value: its descendants get them, others what they had."""
    s = Step([30 + new, 16 + new], [new, new], H, g, D, frozen=frozen, tree=True, seed=6)
    ctx = saf.Context(0)
    s.call(ctx)
    s.check()
    clean = s.O.clone()
    hit = 2
    at = 30 + hit
    page = int(s.table[0, at // 16])
    s.vc[page, :, at % 16, 3] = what
    s.kc[page, :, at % 16] = what
    s.call(ctx)
    torch.cuda.synchronize()
    for i in range(new):
        sees = (s.sets[0][i] >> hit) & 1
        for h in range(H):
            if not sees:
                assert torch.equal(s.O[i, h], clean[i, h]), (i, h)
            elif frozen and s.mask[h]:
                assert not torch.isfinite(s.O[i, h, 3]) and torch.isfinite(s.O[i, h, 4:]).all()
            else:
                assert not torch.isfinite(s.O[i, h]).all()
    assert torch.equal(s.O[new:2 * new], clean[new:2 * new])


def test_preferences_of_minus_infinity_and_of_the_lowest_value():
    s = Step([50, 3], [1, 1], 2, 1, 64, frozen=(0, 1))
    s.alpha[0, 10:40] = float("-inf")
    s.alpha[1, :] = torch.finfo(torch.float32).min
    s.alpha[1, 2] = 0.0
    s.rho[0, 5] = float("-inf")
    s.call_and_check()


def test_lengths_beyond_the_bound_and_rows_beyond_the_count_are_cut():
    s = Step([300, 40], [6, 2], 4, 2, 64, frozen=(3,), max_new=2)
    s.call(saf.Context(0))
    torch.cuda.synchronize()
    assert (s.O[2:6] == 9.0).all() and (s.O[0:2] != 9.0).any() and (s.O[6:8] != 9.0).any()
    # a length beyond max_len counts as max_len
    t = Step([64, 40], [1, 2], 4, 2, 64, frozen=(3,), max_len=64)
    ctx = saf.Context(0)
    t.call(ctx)
    t.check()
    O = t.O.clone()
    t.d_lens[0] = 1000000
    t.call(ctx)
    torch.cuda.synchronize()
    assert torch.equal(O, t.O)


def test_pages_and_rows_out_of_range_reach_nothing():
    """Page numbers outside the pool are clamped, offsets that do not ascend or pass N give no rows: no fault, other requests untouched."""
    s = Step([100, 40, 33], [1, 2, 1], 4, 2, 64, frozen=(3,), poison=0.0)
    ctx = saf.Context(0)
    s.table[0] = torch.tensor([-1, 2 ** 31 - 1, 10 ** 6, -2 ** 31] * 10, dtype=torch.int32, device="cuda")[:s.table.shape[1]]
    s.call(ctx)
    s.check(only=[1, 2])
    assert torch.isfinite(s.O).all()
    s.O.fill_(9.0), s.LSE.fill_(9.0)
    s.d_off.copy_(ints([0, -5, 3, 10 ** 6]))
    s.call(ctx)
    torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """A pool of more than 2^31 elements (and of more than 2^32 bytes): its last pages are read as any others."""
    page, Hk, D = 64, 8, 128
    pages = (2 ** 31 + 2 ** 26) // (page * Hk * D)
    s = Step([200, 100], [1, 2], 16, 2, D, page, "slot", (3,))
    old = s.kc, s.vc
    s.kc, s.vc = (torch.empty((pages, page, Hk, D), device="cuda", dtype=torch.bfloat16).transpose(1, 2) for _ in range(2))
    table = s.table.clone()
    for r in range(2):
        for c in range(-(-s.lens[r] // page)):
            t = pages - 1 - (5 * r + c)
            for new, was in zip((s.kc, s.vc), old):
                new[t] = was[int(table[r, c])]
            s.table[r, c] = t
    s.prob = saf.make_cache(2, s.N, page, pages, s.table.shape[1], k_cache=s.kc, v_cache=s.vc, q_like=s.q, o_like=s.O, Tp=s.alpha.shape[1], max_len=200, max_new=2)
    s.call_and_check()


def test_recorded_steps_serve_other_lengths_and_repeat_bit_for_bit():
    ctx = saf.Context(0)
    s = Step([700, 40, 5000, 9], [3, 2, 1, 1], 8, 4, 64, frozen=(1, 2), max_len=6000, tree=True)
    s.call(ctx)
    s.check()
    first = s.O.clone()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.call(ctx)
    for _ in range(3):
        s.O.fill_(9.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, s.O)
    # shorter contexts in the same arrays
    t = Step([3, 40, 100, 9], [3, 2, 1, 1], 8, 4, 64, frozen=(1, 2), max_len=100, tree=True)
    n = [-(-x // 16) for x in t.lens]
    for r in range(4):
        for c in range(n[r]):
            for pool_s, pool_t in ((s.kc, t.kc), (s.vc, t.vc)):
                pool_s[int(s.table[r, c])] = pool_t[int(t.table[r, c])]
    s.d_lens.copy_(t.d_lens), s.positions.copy_(t.positions), s.masks.copy_(t.masks), s.q.copy_(t.q)
    s.alpha[:, :t.alpha.shape[1]].copy_(t.alpha), s.rho[:, :t.rho.shape[1]].copy_(t.rho)
    s.O.fill_(9.0)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    s.lens, s.k, s.v, s.pos, s.sets = t.lens, t.k, t.v, t.pos, t.sets
    s.check()


def test_two_contexts_on_two_streams():
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Step([4000, 300, 77], [1, 1, 1], 8, 2, 64, frozen=(1,), seed=i) for i in range(2)]
    ctxs = [saf.Context(0) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, s, c in zip(streams, steps, ctxs):
            with torch.cuda.stream(st):
                s.call(c)
    for s in steps:
        s.check()


def test_one_context_serves_calls_of_other_shapes_in_turn():
    ctx = saf.Context(0)
    steps = [Step([900, 30], [1, 1], 8, 2, 64, frozen=(1,)), Step([5000] * 3, [40, 1, 3], 8, 4, 128, frozen=(2,), tree=True), Step([2], [1], 2, 1, 96)]
    for _ in range(3):
        for s in steps:
            s.O.fill_(9.0), s.LSE.fill_(9.0)
            s.call(ctx)
        for s in steps:
            s.check()


def test_attention_refusals():
    ctx = saf.Context(0)

    def refused(code, change=None, stride=None, drop=None, shift=None):
        s = Step([40, 3], [2, 1], 4, 2, 64, frozen=(1,), tree=True)
        if change:
            setattr(s.prob, *change)
        if stride:
            getattr(s.prob, stride[0])[stride[1]] = stride[2]
        a = {"q": s.q, "kc": s.kc, "vc": s.vc, "table": s.table, "off": s.d_off, "lens": s.d_lens, "pos": s.positions, "masks": s.masks, "mask": s.mask,
             "alpha": s.alpha, "rho": s.rho, "O": s.O, "LSE": s.LSE}
        if drop:
            a[drop] = None
        if shift:
            a[shift] = a[shift].flatten()[1:]
        before = s.O.clone()
        with pytest.raises(saf.SafError) as e:
            ctx.saf_cache_attn(s.prob, *a.values())
        assert e.value.code == code
        torch.cuda.synchronize()
        assert torch.equal(before, s.O)

    for change, code in ((("R", 0), 1), (("R", 5000), 1), (("N", 0), 1), (("page_size", 8), 2), (("page_size", 0), 1), (("D", 80), 2), (("D", 256), 2), (("H", 3), 1), (("H", 0), 1),
                         (("kv_group", -2), 1), (("Tp", 10), 1), (("max_new", 0), 1), (("max_new", 65), 1), (("max_len", 0), 1), (("max_len", 1 << 20), 1), (("o_dtype", 7), 2), (("max_pages", 0), 1)):
        refused(code, change=change)
    for name in ("q_strides", "o_strides", "k_strides", "v_strides"):
        refused(1, stride=(name, 0, 12))
        refused(1, stride=(name, 1, -64))
    for name in ("q", "kc", "vc", "table", "off", "lens", "alpha", "rho", "O"):
        refused(1, drop=name)
    for name in ("q", "kc", "vc", "O"):
        refused(1, shift=name)


def _call_and_check(self, only=None):
    self.call(saf.Context(0))
    return self.check(only)


Step.call_and_check = _call_and_check


# ------------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("tree", [False, True])
def test_prompts_then_steps_equal_the_layer(tree):
    """Prompts through plan, append and the layer's own prefill; then tokens (or drafted trees, of which a path is kept) through plan, append
    and attention: every kept token's output equals the row of the square causal layer over the whole sequence."""
    from oracle import saf_oracle as layer
    gen = torch.Generator(device="cuda").manual_seed(9)
    rng = np.random.default_rng(9)
    ctx = saf.Context(0)
    R, H, g, D, page, T = 3, 4, 2, 64, 16, 120
    Hk = H // g
    mask = np.array([0, 1, 0, 0], np.uint8)
    Tp = T + 16                                             # a drafted tree takes more places than positions
    alpha = torch.randn((H, Tp), generator=gen, device="cuda")
    rho = -0.03 * torch.arange(Tp, device="cuda").float() + 0.1 * torch.randn((H, Tp), generator=gen, device="cuda")
    q, k, v = (torch.randn((R, T, h, D), generator=gen, device="cuda").bfloat16() for h in (H, Hk, Hk))
    freqs = saf.saf_rotary_freqs(D)[0]
    f = torch.from_numpy(freqs).cuda()
    turned = [torch.empty_like(t) for t in (q, k)]
    by_head = lambda t: t.transpose(1, 2)  # noqa: E731
    ctx.saf_rotary_fwd(saf.make_rotary(by_head(q), by_head(k), by_head(turned[0]), by_head(turned[1]), D), by_head(q), by_head(k), None, f,
                       by_head(turned[0]), by_head(turned[1]))
    rep = lambda t: np.repeat(f64(by_head(t)), g, axis=1)  # noqa: E731
    want, _ = layer.hybrid_attn_fwd(f64(by_head(turned[0])), rep(turned[1]), rep(v), mask, f64(alpha[:, :T]), f64(rho[:, :T]))
    kc, vc = pool(40, Hk, page, D, "page", float("nan")), pool(40, Hk, page, D, "page", float("nan"))
    s = Pages(R, 256, page, 40, Tp // page + 2)
    drafts = Pages(R, 256, page, 40, Tp // page + 2, tree=True)
    state = (s.d_held, s.d_count, s.d_free, s.d_table)
    lens = [0] * R
    step = 0
    while min(lens) < T - 8:
        if step == 0:
            path = [[int(x) for x in range(n)] for n in (17, 60, 1)]      # prompts, as chains
            new, parents = [len(p) for p in path], None
        elif tree:
            # each request: a path of tokens to come, with wrong ones (tokens of other places) between
            new, parents, path, tokens = [], [], [], []
            for r in range(R):
                good, par, tok = [], [], []
                for d in range(min(4, T - lens[r])):
                    for _ in range(int(rng.integers(0, 3))):
                        par.append(good[-1] if good else -1), tok.append(int(rng.integers(0, T)))
                    par.append(good[-1] if good else -1), tok.append(lens[r] + d)
                    good.append(len(par) - 1)
                new.append(len(par)), parents.append(par), path.append(good), tokens.append(tok)
        else:
            new, parents = [1 + step % 2] * R, None
            new = [min(n, T - x) for n, x in zip(new, lens)]
            path = [list(range(n)) for n in new]
        p = drafts if parents is not None else s
        p.d_held, p.d_count, p.d_free, p.d_table = state
        total = sum(new)
        flat = None if parents is None else ints(sum(parents, []) + [0] * (256 - total))
        p.device(ctx, ints(lens), ints(new), flat)
        rows = sum(([(r, lens[r] + i if parents is None else tokens[r][i]) for i in range(new[r])] for r in range(R)), [])
        rr, tt = (torch.tensor([x[i] for x in rows], device="cuda") for i in range(2))
        qn, kn, vn = (torch.zeros((256, t.shape[2], D), device="cuda", dtype=torch.bfloat16) for t in (q, k, v))
        qn[:total], kn[:total], vn[:total] = q[rr, tt], k[rr, tt], v[rr, tt]
        qo, O = torch.zeros_like(qn), torch.zeros((256, H, D), device="cuda", dtype=torch.bfloat16)
        c = saf.make_cache(R, 256, page, 40, s.max_pages, k_cache=kc, v_cache=vc, v_like=vn)
        ctx.saf_cache_append(c, saf.make_rotary(qn, kn, qo, None, D), qn, kn, vn, p.out["slots"], p.out["positions"], f, qo, kc, vc)
        if step > 0:
            c = saf.make_cache(R, 256, page, 40, s.max_pages, k_cache=kc, v_cache=vc, q_like=qo, o_like=O, Tp=Tp, max_len=Tp, max_new=64)
            ctx.saf_cache_attn(c, qo, kc, vc, p.d_table, p.out["offsets"], p.out["kv_lens"], p.out["positions"], p.masks if parents is not None else None, mask,
                               alpha, rho, O, None)
            torch.cuda.synchronize()
            at = 0
            for r in range(R):
                for d, i in enumerate(path[r]):
                    # (the bound of the layer's parity tests; keys and queries are the same bf16 values)
                    assert np.abs(f64(O[at + i]) - want[r, :, lens[r] + d]).max() <= 2e-2
                at += new[r]
        # the accepted path moves to the places behind the context
        for r in range(R):
            tab = p.d_table[r]
            for d, i in enumerate(path[r]):
                src, dst = lens[r] + i, lens[r] + d
                if src != dst:
                    for cache in (kc, vc):
                        cache[tab[dst // page], :, dst % page] = cache[tab[src // page], :, src % page].clone()
        lens = [x + len(g_) for x, g_ in zip(lens, path)]
        state = (p.d_held, p.d_count, p.d_free, p.d_table)
        step += 1
    torch.cuda.synchronize()
    assert ctx.saf_last_device_status()[0] == saf.SAF_OK


# ------------------------------------------------------------------------------------------------------------------- many rows
@pytest.mark.parametrize("H,g,D,frozen", GEOMETRY)
def test_many_rows_of_fp32(H, g, D, frozen):
    Step([500, 64, 17, 333], [40, 64, 17, 3], H, g, D, 32, "slot", frozen, tree=True, out="fp32", seed=7).call_and_check()


# frozen heads of a group: as many as have two places each, up to twice as many, and more than have one
@pytest.mark.parametrize("nf", [1, 5, 6, 7, 12, 13, 16])
@pytest.mark.parametrize("D,page,layout", [(64, 128, "page"), (96, 48, "slot"), (128, 16, "page")])
@pytest.mark.parametrize("tree", [False, True])
def test_frozen_heads_of_one_group(nf, D, page, layout, tree):
    frozen = tuple(np.random.default_rng(nf).permutation(16)[:nf]) + tuple(16 + i for i in range(0, 16, 3))
    Step([700, 9, 130, 65], [9, 9, 2, 1], 32, 16, D, page, layout, frozen, tree=tree, seed=nf).call_and_check()


@pytest.mark.parametrize("H,g,D,new", [(100, 100, 64, [3, 1, 2]), (128, 128, 128, [1, 2, 1]), (130, 65, 96, [2, 3, 1]), (129, 129, 64, [2, 1, 1]), (512, 256, 64, [1, 1, 1])])
def test_groups_of_many_heads(H, g, D, new):
    frozen = tuple(range(0, H, 17))
    Step([300, 3, 65], new, H, g, D, 16, "page", frozen, seed=8).call_and_check()


@pytest.mark.parametrize("D,g", [(64, 2), (96, 4), (128, 1)])
@pytest.mark.parametrize("ctx", [0, 1, 23, 24, 25, 63, 64, 65, 87, 88, 89])
def test_many_rows_at_the_edges_of_tiles(D, g, ctx):
    new = [40, 41, 39, 0, 64]
    Step([ctx + n for n in new], new, 2 * g, g, D, 16, "page", (0,), tree=ctx % 2 == 0, seed=ctx).call_and_check()


@pytest.mark.parametrize("D,g,frozen,page,layout", [(64, 2, (1, 2), 128, "slot"), (96, 2, (), 48, "page"), (128, 4, tuple(range(8)), 64, "slot"), (128, 2, (0, 3), 16, "page")])
@pytest.mark.parametrize("lens", [[5000, 64, 700], [9000], [64] * 150 + [4000], [1000, 0, 2500, 64, 5999]])
def test_many_rows_split_over_blocks(D, g, frozen, page, layout, lens):
    new = [0 if n == 0 else 33 if i % 2 else 64 for i, n in enumerate(lens)]
    only = range(0, len(lens), 29) if len(lens) > 100 else None
    Step(lens, new, 2 * g, g, D, page, layout, frozen, tree=True, seed=9).call_and_check(only)


@pytest.mark.parametrize("D,g,new", [(64, 4, 5), (64, 4, 40), (96, 2, 40), (128, 2, 6), (128, 4, 40)])
def test_positions_anywhere(D, g, new):
    """New tokens whose positions neither ascend nor stay near their places."""
    s = Step([new + 300, new, new + 70], [new] * 3, 2 * g, g, D, 16, "page", (0, g), tree=True, seed=10)
    rng = np.random.default_rng(11)
    s.pos = [rng.integers(0, s.max_len, new) for _ in range(3)]
    s.positions = ints([int(x) for p in s.pos for x in p] + [-9] * 2)
    s.call_and_check()


def test_positions_out_of_range_are_clamped():
    for g, new in ((1, 4), (4, 40)):
        s = Step([new + 30], [new], 2 * g, g, 128, 16, "page", (0,), tree=True, seed=12)
        last = s.alpha.shape[1] - 1
        s.pos = [np.array([0, last, 7, last] * (new // 4))]
        s.positions = ints([-2 ** 31, 2 ** 31 - 1, 7, last + 1] * (new // 4) + [-9] * 2)
        s.call_and_check()


def test_many_rows_of_slices_scale_and_no_lse():
    s = Step([170, 33], [33, 21], 8, 4, 128, 32, "slot", (1, 4), sliced=True, scale=0.07, positions=False)
    s.call_and_check()
    O = s.O.clone()
    s.O.fill_(9.0)
    s.call(saf.Context(0), lse=False)
    assert torch.equal(O, s.O)


@pytest.mark.parametrize("D", [64, 128])
def test_many_rows_that_see_nothing_or_lie_out_of_range(D):
    ctx = saf.Context(0)
    s = Step([40, 300, 90], [40, 33, 20], 4, 2, D, frozen=(1,), tree=True, poison=0.0)
    s.masks[1] = 0
    s.d_lens[2] = 0
    s.call(ctx)
    s.check(only=[1])
    assert not s.O[1].any() and s.O[0].any() and not s.O[73:93].any()
    assert (s.LSE[73:93, [0, 2, 3]] == float("-inf")).all() and not s.LSE[73:93, 1].any() and (s.LSE[1, [0, 2, 3]] == float("-inf")).all()
    # page numbers outside the pool, and offsets that do not ascend or pass N
    s = Step([400, 140, 33], [40, 32, 33], 4, 2, D, frozen=(3,), tree=True, poison=0.0)
    s.table[0] = torch.tensor([-1, 2 ** 31 - 1, 10 ** 6, -2 ** 31] * 10, dtype=torch.int32, device="cuda")[:s.table.shape[1]]
    s.call(ctx)
    s.check(only=[1, 2])
    assert torch.isfinite(s.O).all()
    s.d_off.copy_(ints([0, -5, 3, 10 ** 6]))
    s.call(ctx)
    # more rows than max_new, more tokens than max_len
    s = Step([300, 90], [40, 34], 4, 2, D, frozen=(3,), max_new=34)
    s.call(ctx)
    torch.cuda.synchronize()
    assert (s.O[34:40] == 9.0).all() and (s.O[33] != 9.0).any() and (s.O[40:74] != 9.0).any()
    s.d_lens[1] = 1000000
    s.call(ctx)
    torch.cuda.synchronize()


def test_many_rows_and_preferences_of_minus_infinity_and_of_the_lowest_value():
    s = Step([150, 40], [33, 40], 4, 4, 64, frozen=(0, 1, 3), tree=True)
    s.alpha[0, 10:140] = float("-inf")
    s.alpha[1, :] = torch.finfo(torch.float32).min
    s.alpha[1, 2] = 0.0
    s.rho[0, 5] = float("-inf")
    s.call_and_check()


def test_recorded_steps_of_many_rows_on_another_stream():
    ctx = saf.Context(0)
    s = Step([7000, 140, 5000, 39], [33, 40, 21, 39], 8, 4, 128, frozen=(1, 2), tree=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.call(ctx)
    s.check()
    first = s.O.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        s.call(ctx)
    for _ in range(3):
        s.O.fill_(9.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, s.O)
    s.check()


def test_one_context_serves_few_and_many_rows_in_turn():
    ctx = saf.Context(0)
    steps = [Step([900, 4000], [1, 1], 8, 2, 128, frozen=(1,)), Step([5000] * 3, [40, 1, 3], 8, 4, 128, frozen=(2,), tree=True),
             Step([3000], [40], 4, 2, 64, out="fp32"), Step([6000, 65], [64, 64], 4, 2, 64, frozen=(0,)), Step([2], [1], 2, 1, 96)]
    for _ in range(3):
        for s in steps:
            s.O.fill_(9.0), s.LSE.fill_(9.0)
            s.call(ctx)
        for s in steps:
            s.check()


def test_more_tiles_than_32_bits_are_refused():
    s = Step([40, 3], [2, 1], 4, 2, 64, frozen=(1,))
    for R, H, g, max_new in ((4096, 1024, 1, 16), (4096, 1024, 1, 64), (4096, 1024, 8, 64)):
        s.prob.R, s.prob.H, s.prob.kv_group, s.prob.max_new = R, H, g, max_new
        s.prob.page_size, s.prob.max_pages, s.prob.max_len, s.prob.Tp = 1 << 18, 1 << 8, 1 << 26, 1 << 26
        with pytest.raises(saf.SafError) as e:
            s.call(saf.Context(0))
        assert e.value.code == 2
    s.prob.R = s.prob.H = s.prob.kv_group = s.prob.max_new = 1           # lengths whose tiles would end beyond 2^31
    s.prob.max_pages, s.prob.page_size, s.prob.max_len = 2 ** 24 - 1, 128, 2 ** 31 - 128
    with pytest.raises(saf.SafError) as e:
        s.call(saf.Context(0))
    assert e.value.code == 2
    torch.cuda.synchronize()


def test_recorded_step_after_a_larger_call():
    """The workspace of a recorded call stays where it is when calls with more rows and wider heads follow."""
    ctx = saf.Context(0)
    s = Step([4000, 300, 77], [1, 1, 1], 8, 2, 64, frozen=(1,))
    s.call(ctx)
    s.check()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        s.call(ctx)
    for other in (Step([5000], [40], 4, 2, 128, out="fp32"), Step([3000, 400], [64, 33], 8, 4, 128, frozen=(2,), tree=True)):
        other.call(ctx)
        other.check()
        s.O.fill_(9.0), s.LSE.fill_(9.0)
        torch.cuda.synchronize()
        g.replay()
        s.check()


def test_two_contexts_of_many_rows_on_two_streams():
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Step([4000, 300, 77], [40, 33, 64], 8, 4, 128, frozen=(1,), tree=True, seed=i) for i in range(2)]
    ctxs = [saf.Context(0) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, s, c in zip(streams, steps, ctxs):
            with torch.cuda.stream(st):
                s.call(c)
    for s in steps:
        s.check()


@pytest.mark.parametrize("D,g,new,out", [(64, 2, 1, "bf16"), (128, 4, 3, "fp32"), (128, 4, 40, "bf16")])
def test_the_same_call_twice_gives_the_same_bits(D, g, new, out):
    ctx = saf.Context(0)
    s = Step([9000, 1200, 65], [new] * 3, 2 * g, g, D, 16, "page", (0,), tree=True, out=out, seed=13)
    s.call(ctx)
    torch.cuda.synchronize()
    O, L = s.O.clone(), s.LSE.clone()
    for c in (ctx, saf.Context(0)) * 5:
        s.O.fill_(9.0), s.LSE.fill_(9.0)
        s.call(c)
        torch.cuda.synchronize()
        assert torch.equal(O, s.O) and torch.equal(L, s.LSE)
