"""Measured cases of the operators that serve a hybrid layer from a paged key/value cache, and of the rotary positions that
training shares with it.

`op` says which operator a case is:

  plan     pages given to and taken from requests by their lengths, and what the other calls need to know of one step: first
           row of each request, slot and position of each new token, ancestor sets of drafted trees
  rotary   rotary positions on queries and keys; `back` adds the gradients' way back
  append   a step's new tokens: queries and keys rotated, keys and values written to their slots of the cache
  attend   attention of a step's new tokens (one a request, a short chain, a drafted tree) over the cache, ordinary and frozen
           heads side by side

Lengths are spread evenly over their range and dealt to the requests in an order that the seed draws; which heads are frozen
goes by the case, as in a model.
"""
import functools
import math
import random

import torch

own = False

PLAN, ROTARY, APPEND, ATTEND = "plan", "rotary", "append", "attend"


# --------------------------------------------------------------------------------------------------- the cases
def _plan(R, ctx, new, page, tree=False, short=False):
    return {"op": PLAN, "R": R, "ctx": ctx, "new": new, "page": page, "tree": tree, "short": short}


def _rotary(B, H, group, T, D, rot, interleaved, scaling="none", back=False, grads="fp32", out="bf16", layout="bthd"):
    return {"op": ROTARY, "B": B, "H": H, "group": group, "T": T, "D": D, "rot": rot, "interleaved": interleaved,
            "scaling": scaling, "back": back, "grads": grads, "out": out, "layout": layout}


def _append(R, ctx, new, H, group, D, rot, page, layout="page"):
    return {"op": APPEND, "R": R, "ctx": ctx, "new": new, "H": H, "group": group, "D": D, "rot": rot, "page": page, "layout": layout}


def _attend(R, ctx, new, H, group, D, frozen, page, tree=False, out="bf16", layout="page"):
    return {"op": ATTEND, "R": R, "ctx": ctx, "new": new, "H": H, "group": group, "D": D, "frozen": frozen, "page": page,
            "tree": tree, "out": out, "layout": layout}


def listed():
    return [
        # one decoding step of 64 requests, one token each: latency between two steps
        dict(_plan(64, 4096, 1, 16), name="plan-decode"),
        # a step of 256 requests that verify drafted trees; some have just ended and give their pages back
        dict(_plan(256, 32768, 32, 16, tree=True), name="plan-trees"),
        # queries and keys of the smallest test configuration and their gradients: latency
        dict(_rotary(1, 4, 1, 256, 64, 64, False, back=True, out="fp32", layout="bhtd"), name="rotary-tiny"),
        # the 124M layer's training update (12 heads x 64, 4K context, batch 8): fp32 gradients back to bf16
        dict(_rotary(8, 12, 1, 4096, 64, 64, False, back=True), name="rotary-update-124m"),
        # long-context prefill on grouped-query heads (32 on 8, dimension 128): interleaved pairs, three quarters of a head,
        # frequencies stretched for the long context
        dict(_rotary(1, 32, 4, 32768, 128, 96, True, scaling="ramp"), name="rotary-prefill-32k"),
        # a decoding step of 64 requests on grouped-query heads
        dict(_append(64, 4096, 1, 32, 4, 128, 128, 16), name="append-decode"),
        # ragged prompts of a batch of 32 enter the cache of a 1B-shaped layer (16 heads x 96)
        dict(_append(32, 0, 1537, 16, 1, 96, 96, 64, layout="slot"), name="append-prompts"),
        # one user's next token on the 124M layer, 25 % frozen: launch and latency
        dict(_attend(1, 200, 1, 12, 1, 64, 3, 16), name="attend-one-user"),
        # decoding batch on the 124M layer
        dict(_attend(32, 4096, 1, 12, 1, 64, 3, 16), name="attend-decode-124m"),
        # decoding batch with long contexts on grouped-query heads, 30 % frozen
        dict(_attend(16, 32768, 1, 32, 4, 128, 10, 64, layout="slot"), name="attend-gqa-32k"),
        # drafted trees of up to 32 tokens verified on grouped-query heads
        dict(_attend(24, 8192, 32, 32, 4, 128, 10, 16, tree=True), name="attend-trees"),
        # chains of up to five drafted tokens on the paper's 1B layer (16 heads x 96), fp32 output
        dict(_attend(8, 8192, 5, 16, 1, 96, 4, 32, out="fp32"), name="attend-chains-d96"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges."""
    op = rng.choice([PLAN, ROTARY, APPEND] + [ATTEND] * 4)
    page = rng.choice([16, 32, 64, 128])
    layout = rng.choice(["page", "slot"])
    if op == PLAN:
        tree = rng.random() < 0.5
        new = _log_uniform(rng, 2, 64) if tree else rng.choice([1, 1, _log_uniform(rng, 2, 512)])
        return _plan(_log_uniform(rng, 1, 256), _log_uniform(rng, 1, 32768), new, page, tree, rng.random() < 0.2)
    H, group, D = rng.choice([(12, 1, 64), (32, 1, 64), (16, 4, 64), (16, 1, 96), (12, 1, 128), (32, 4, 128), (16, 8, 128)])
    rot = rng.choice([D, D, D // 2])
    if op == ROTARY:
        T = _log_uniform(rng, 1, 32768)
        B = _log_uniform(rng, 1, max(1, min(16, 32768 // T)))
        if H * T * B * D > 8 * 12 * 4096 * 64:
            B, T = 1, 4096
        return _rotary(B, H, group, T, D, rot, rng.random() < 0.5, rng.choice(["none", "ramp"]), rng.random() < 0.5,
                       rng.choice(["fp32", "bf16"]), rng.choice(["bf16", "bf16", "fp32"]), rng.choice(["bthd", "bhtd"]))
    R, ctx = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 32768)
    if op == APPEND:
        new = rng.choice([1, 1, _log_uniform(rng, 2, 1537)])
        R = min(R, 32) if new > 1 else R
        # the pool holds what the requests hold, and the listed cases' pools are not exceeded
        ctx = max(1, min(ctx, 32 * 1537 * 16 * 96 // (R * D * (H // group)) - new))
        return _append(R, ctx, new, H, group, D, rot, page, layout)
    kind = rng.choice(["one", "one", "chain", "tree"])
    new = 1 if kind == "one" else _log_uniform(rng, 2, 8) if kind == "chain" else _log_uniform(rng, 2, 64)
    # no more keys, and no more scores, than the largest listed cases have
    ctx = max(1, min(ctx, 16 * 32768 * 8 * 128 // (R * D * (H // group)), 24 * 8192 * 32 * 32 // (R * new * H)))
    frozen = int(round(H * rng.choice([0.0, 0.25, 0.25, 0.5, 1.0])))
    return _attend(R, ctx, new, H, group, D, frozen, page, kind == "tree", rng.choice(["bf16", "bf16", "fp32"]), layout)


# --------------------------------------------------------------------------------------------------- inputs
def _spread(n, lo, hi):
    """n lengths evenly over [lo, hi]."""
    return [lo + int((hi - lo) * (i + 0.5) / n + 0.5) for i in range(n)]


def _lengths(case):
    """(tokens in the cache, new tokens) of every request, before the seed deals them out."""
    R, new = case["R"], case["new"]
    ctx = _spread(R, case["ctx"] // 64, case["ctx"]) if R > 1 else [case["ctx"]]
    many = [1] * R if new == 1 else _spread(R, max(1, new // 4), new) if R > 1 else [new]
    many = [many[i * 7 % R] if R % 7 else many[i] for i in range(R)]
    if case["op"] == PLAN and R >= 8:                      # one in eight has ended: no tokens, no pages
        ctx, many = [c if i % 8 else 0 for i, c in enumerate(ctx)], [n if i % 8 else 0 for i, n in enumerate(many)]
    return ctx, many


def _frozen(case):
    """Which heads are frozen: by the case alone, as in a model."""
    chosen = set(random.Random(1000).sample(range(case["H"]), case["frozen"]))
    return [1 if h in chosen else 0 for h in range(case["H"])]


def _requests(case, gen):
    ctx, many = _lengths(case)
    order = torch.randperm(case["R"], generator=gen, device="cuda").cpu().tolist()
    ctx, many = [ctx[i] for i in order], [many[i] for i in order]
    return torch.tensor(ctx, dtype=torch.int32, device="cuda"), torch.tensor(many, dtype=torch.int32, device="cuda")


def _offsets(new):
    return torch.cat([new.new_zeros(1), new.cumsum(0).int()])


def _rows(s):
    """(request, place within it) of every packed row; rows behind the last request have request R."""
    rows = torch.arange(s["N"], device="cuda")
    offs = s["offsets"].long()
    r = torch.searchsorted(offs[1:].contiguous(), rows, right=True)
    return r, rows - offs[r.clamp(max=s["R"] - 1)]


def _parents(place, gen):
    """A random tree a request: each drafted token follows one before it, or the last cached one (-1)."""
    u = torch.rand(place.shape, generator=gen, device="cuda")
    return torch.minimum((u * (place + 1)).long(), place).int() - 1


def _ancestors(parents, r, place, R):
    """Ancestor sets, the token itself in them, as bits; and depths.  In a forest the (i, j) entry of (1 + A)^64 is not zero
    exactly where j lies on i's way up."""
    up = torch.zeros((R + 1, 64, 64), dtype=torch.float64, device=parents.device)
    has = parents >= 0
    up[r[has], place[has], parents[has].long()] = 1.0
    reach = torch.matrix_power(up + torch.eye(64, dtype=torch.float64, device=up.device), 64) > 0
    sets = reach[r, place.clamp(0, 63)]
    bits = (sets.long() << torch.arange(64, device=up.device)).sum(1)
    return bits, sets.sum(1) - 1


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _heads(gen, B, H, T, D, layout, dtype=torch.bfloat16):
    """[B,H,T,D], in memory as projections leave it ("bthd") or head by head."""
    if layout == "bthd":
        return torch.randn((B, T, H, D), generator=gen, device="cuda").to(dtype).transpose(1, 2)
    return torch.randn((B, H, T, D), generator=gen, device="cuda").to(dtype)


def _pool(gen, pages, heads, page, D, layout):
    """Cache [pages, heads, page, D]: head by head within a page ("page"), or slot by slot ("slot")."""
    if layout == "slot":
        return _normal(gen, pages, page, heads, D).transpose(1, 2)
    return _normal(gen, pages, heads, page, D)


def _frequencies(rot, scaling):
    """Radians per position, in 64 bits.  "ramp": eight times the trained context of 4096, slow pairs divided by the factor, fast
    ones left, a linear ramp between 32 and 1 turns over the trained context, outputs scaled by 0.1 ln 8 + 1."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "none":
        return f.cuda(), 1.0

    def pair(turns):
        return rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
    lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
    keep = 1.0 - ((torch.arange(rot // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
    return (f / 8.0 * (1 - keep) + f * keep).cuda(), 0.1 * math.log(8.0) + 1.0


def _prepare_plan(case, gen):
    R, page = case["R"], case["page"]
    s = {"op": PLAN, "R": R, "page": page, "tree": case["tree"]}
    ctx, many = _lengths(case)
    s["ctx"], s["new"] = _requests(case, gen)
    s["N"] = sum(many) + 3                                # a step's arrays are a little larger than the step, as in a graph
    s["max_pages"] = -(-(case["ctx"] + case["new"]) // page) + 1
    pages = sum(-(-(c + n) // page) for c, n in zip(ctx, many)) + 4 * R
    # before the step a request holds what its cached tokens take; every fifth holds a drafted tail that was not accepted,
    # and those that have ended hold some pages still
    held = (s["ctx"].long() + page - 1) // page
    idle = s["new"] == 0
    held = torch.where(torch.arange(R, device="cuda") % 5 == 0, held + 2, held)
    held = torch.where(idle, torch.full_like(held, 3), held).clamp(max=s["max_pages"])
    ids = torch.randperm(pages + 5 * R, generator=gen, device="cuda").int()
    s["pages"] = ids.numel()
    col = torch.arange(s["max_pages"], device="cuda")
    taken = col[None, :] < held[:, None]
    s["table"] = torch.zeros((R, s["max_pages"]), dtype=torch.int32, device="cuda")
    s["table"][taken] = ids[:int(held.sum())]
    s["held"] = held.int()
    rest = ids[int(held.sum()):]
    s["free"] = torch.cat([rest, torch.full((s["pages"] - rest.numel(),), -1, dtype=torch.int32, device="cuda")])
    count = 1 if case["short"] else rest.numel()           # "short": the pool runs out
    s["count"] = torch.tensor([count], dtype=torch.int32, device="cuda")
    s["offsets"] = _offsets(s["new"])
    if case["tree"]:
        r, place = _rows(s)
        s["parents"] = torch.where(r < R, _parents(place.clamp(min=0), gen), -1).int()
    s["out"] = {"held": torch.empty_like(s["held"]), "count": torch.empty_like(s["count"]), "offsets": torch.empty_like(s["offsets"]),
                "kv_lens": torch.empty_like(s["ctx"]), "missing": torch.empty_like(s["ctx"]),
                "slots": torch.empty(s["N"], dtype=torch.int32, device="cuda"), "positions": torch.empty(s["N"], dtype=torch.int32, device="cuda")}
    if case["tree"]:
        s["out"]["masks"] = torch.empty(s["N"], dtype=torch.int64, device="cuda")
    return s


def _prepare_rotary(case, gen):
    B, H, T, D, g = case["B"], case["H"], case["T"], case["D"], case["group"]
    s = {"op": ROTARY, "rot": case["rot"], "interleaved": case["interleaved"], "back": case["back"]}
    out = torch.float32 if case["out"] == "fp32" else torch.bfloat16
    grad = torch.float32 if case["grads"] == "fp32" else torch.bfloat16
    s["q"], s["k"] = _heads(gen, B, H, T, D, case["layout"]), _heads(gen, B, H // g, T, D, case["layout"])
    s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    # each sequence starts somewhere in a document of its own
    start = torch.randint(0, 4096, (B, 1), generator=gen, device="cuda")
    s["positions"] = (start + torch.arange(T, device="cuda")).int().contiguous()
    s["freqs"], s["mscale"] = _frequencies(case["rot"], case["scaling"])
    if case["back"]:
        # the layer's gradients come head by head, contiguous
        s["dq"], s["dk"] = _heads(gen, B, H, T, D, "bhtd", grad), _heads(gen, B, H // g, T, D, "bhtd", grad)
        s["dq_out"] = torch.empty_like(s["q"], dtype=out)
        s["dk_out"] = torch.empty_like(s["k"], dtype=out)
    return s


def _prepare_pages(case, gen, s):
    """Lengths, packed rows and a block table whose pages lie anywhere in the pool."""
    R, page = case["R"], case["page"]
    ctx, many = _lengths(case)
    s["R"], s["page"] = R, page
    s["ctx"], s["new"] = _requests(case, gen)
    s["N"] = sum(many)
    s["offsets"], s["kv_lens"] = _offsets(s["new"]), s["ctx"] + s["new"]
    s["max_len"] = max(c + n for c, n in zip(ctx, [max(many)] * R))
    s["max_new"] = max(many)
    s["max_pages"] = -(-s["max_len"] // page)
    need = (s["kv_lens"].long() + page - 1) // page
    s["pages"] = int(need.sum()) + R
    ids = torch.randperm(s["pages"], generator=gen, device="cuda").int()
    s["table"] = torch.zeros((R, s["max_pages"]), dtype=torch.int32, device="cuda")
    s["table"][torch.arange(s["max_pages"], device="cuda")[None, :] < need[:, None]] = ids[:int(need.sum())]
    r, place = _rows(s)
    s["row_request"], s["row_place"] = r, place
    s["positions"] = (s["ctx"].long()[r] + place).int()
    where = s["ctx"].long()[r] + place
    s["slots"] = (s["table"].long()[r, where // page] * page + where % page).int()


def _prepare_append(case, gen):
    H, D, g = case["H"], case["D"], case["group"]
    s = {"op": APPEND, "rot": case["rot"], "H": H, "group": g, "D": D, "interleaved": False}
    _prepare_pages(case, gen, s)
    # one projection's output: queries, keys and values of a token side by side
    qkv = _normal(gen, s["N"], H + 2 * (H // g), D)
    s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + H // g], qkv[:, H + H // g:]
    s["q_out"] = torch.empty((s["N"], H, D), dtype=torch.bfloat16, device="cuda")
    s["k_cache"], s["v_cache"] = (_pool(gen, s["pages"], H // g, s["page"], D, case["layout"]) for _ in range(2))
    s["freqs"], s["mscale"] = _frequencies(case["rot"], "none")
    return s


def _prepare_attend(case, gen):
    H, D, g = case["H"], case["D"], case["group"]
    s = {"op": ATTEND, "H": H, "group": g, "D": D, "mask": _frozen(case), "tree": case["tree"]}
    _prepare_pages(case, gen, s)
    s["q"] = _normal(gen, s["N"], H, D)
    s["k_cache"], s["v_cache"] = (_pool(gen, s["pages"], H // g, s["page"], D, case["layout"]) for _ in range(2))
    # structured-random key preferences, distance preferences that decay with noise
    L = s["max_len"]
    s["alpha"] = torch.randn((H, L), generator=gen, device="cuda")
    s["rho"] = -0.01 * torch.arange(L, device="cuda").float() + 0.1 * torch.randn((H, L), generator=gen, device="cuda")
    s["masks"] = None
    if case["tree"]:
        r, place = s["row_request"], s["row_place"]
        s["masks"], depth = _ancestors(_parents(place, gen), r, place, s["R"])
        s["positions"] = (s["ctx"].long()[r] + depth).int()
    s["O"] = torch.empty((s["N"], H, D), dtype=torch.float32 if case["out"] == "fp32" else torch.bfloat16, device="cuda")
    s["LSE"] = torch.empty((s["N"], H), device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {PLAN: _prepare_plan, ROTARY: _prepare_rotary, APPEND: _prepare_append, ATTEND: _prepare_attend}[case["op"]](case, gen)


# --------------------------------------------------------------------------------------------------- plain forms
def _plain_plan(s):
    R, N, page, out = s["R"], s["N"], s["page"], s["out"]
    ctx, new, held = s["ctx"].long(), s["new"].long(), s["held"].long()
    need = (ctx + new + page - 1) // page
    ends = new.cumsum(0)
    bad = (need > s["max_pages"]) | (ends > N) & (new > 0)
    if s["tree"]:
        bad = bad | (new > 64)
    need = torch.where(bad, held, need)
    grow, trim = (need - held).clamp(min=0), (held - need).clamp(min=0)
    col = torch.arange(s["max_pages"], device=ctx.device)
    # the free stack, and on it the pages that requests give back, in order of requests and of places
    back = s["table"][(col[None, :] >= need[:, None]) & (col[None, :] < held[:, None])]
    count = s["count"].long()
    given = trim.sum()
    stack = torch.arange(s["free"].numel(), device=ctx.device)
    at = stack - count
    stack = torch.where(at < 0, s["free"], torch.cat([back, back.new_zeros(1)])[at.clamp(0, back.numel())])
    total = count + given
    cum = grow.cumsum(0)
    served = (grow == 0) | (cum <= total)
    taken = torch.where(served, grow, 0).sum()
    ok = served & ~bad
    fill = ok[:, None] & (col[None, :] >= held[:, None]) & (col[None, :] < need[:, None])
    rank = total - 1 - ((cum - grow)[:, None] + col[None, :] - held[:, None])
    s["table"].copy_(torch.where(fill, stack[rank.clamp(0, stack.numel() - 1)], s["table"]))
    left = total - taken
    place = torch.arange(stack.numel(), device=ctx.device)
    s["free"].copy_(torch.where((place >= count) & (place < left), stack, s["free"]))
    out["held"].copy_(torch.where(ok, need, held))
    out["count"].copy_(left)
    out["missing"].copy_(torch.where(bad, -1, torch.where(served, 0, grow)))
    out["kv_lens"].copy_(torch.where(ok, ctx + new, 0))
    out["offsets"].copy_(torch.cat([ends.new_zeros(1), ends.clamp(max=N)]))
    rows = torch.arange(N, device=ctx.device)
    r = torch.searchsorted(ends, rows, right=True)
    here, rr = r < R, r.clamp(max=R - 1)
    i = rows - (ends - new)[rr]
    where = ctx[rr] + i
    slot = s["table"].long()[rr, (where // page).clamp(max=s["max_pages"] - 1)] * page + where % page
    out["slots"].copy_(torch.where(here & ok[rr], slot, -1))
    depth = i
    if s["tree"]:
        fits = here & (new[rr] <= 64)
        line = torch.where(fits, r, R)
        i64 = torch.where(fits, i, 0)
        up = torch.where(fits & (s["parents"] < i64), s["parents"], -1)
        bits, depth = _ancestors(up, line, i64, R)
        out["masks"].copy_(torch.where(fits, bits, 0))
        depth = torch.where(fits, depth, 0)
    out["positions"].copy_(torch.where(here, ctx[rr] + depth, 0))
    return {**out, "table": s["table"], "free": s["free"]}


def _cos_sin(s, positions, sign=1.0):
    # far positions: angles in 64 bits
    angle = positions.double()[..., None] * s["freqs"]
    return (angle.cos() * s["mscale"]).float(), (angle.sin() * (s["mscale"] * sign)).float()


def _turn(x, cos, sin, rot, interleaved):
    """Pairs (2i, 2i + 1), or (i, i + rot / 2), of the first `rot` features turned; in fp32."""
    x = x.float()
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :rot // 2], head[..., rot // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, rest], -1)


def _plain_rotary(s):
    cos, sin = _cos_sin(s, s["positions"])
    cos, sin = cos[:, None], sin[:, None]
    out = {"q": s["q_out"].copy_(_turn(s["q"], cos, sin, s["rot"], s["interleaved"])),
           "k": s["k_out"].copy_(_turn(s["k"], cos, sin, s["rot"], s["interleaved"]))}
    if s["back"]:
        out["dq"] = s["dq_out"].copy_(_turn(s["dq"], cos, -sin, s["rot"], s["interleaved"]))
        out["dk"] = s["dk_out"].copy_(_turn(s["dk"], cos, -sin, s["rot"], s["interleaved"]))
    return out


def _plain_append(s):
    cos, sin = _cos_sin(s, s["positions"])
    cos, sin = cos[:, None], sin[:, None]
    s["q_out"].copy_(_turn(s["q"], cos, sin, s["rot"], s["interleaved"]))
    slots = s["slots"].long()
    page, place = slots // s["page"], slots % s["page"]
    s["k_cache"][page, :, place] = _turn(s["k"], cos, sin, s["rot"], s["interleaved"]).bfloat16()
    s["v_cache"][page, :, place] = s["v"]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    R, H, g, D, L, n = s["R"], s["H"], s["group"], s["D"], s["max_len"], s["max_new"]
    dev = s["q"].device
    r, i = s["row_request"], s["row_place"]
    ctx, lens = s["ctx"].long(), s["kv_lens"].long()
    j = torch.arange(L, device=dev)
    page = s["table"].long()[:, j // s["page"]]
    k = s["k_cache"][page, :, j % s["page"]].float()                                # [R, L, Hkv, D]
    v = s["v_cache"][page, :, j % s["page"]].float()
    v = torch.where((j < lens[:, None])[:, :, None, None], v, 0.0)
    q = s["q"].new_zeros((R, n, H, D)).float()
    q[r, i] = s["q"].float()
    q = q.view(R, n, H // g, g, D).permute(0, 2, 1, 3, 4).reshape(R, H // g, n * g, D)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(D)                  # [R, Hkv, n g, L]
    scores = scores.view(R, H // g, n, g, L).permute(0, 2, 1, 3, 4).reshape(R, n, H, L)
    # which keys a new token sees, and where keys and queries stand
    back = j[None, :] - ctx[:, None]                                                # place among the new tokens
    bits = torch.zeros((R, n), dtype=torch.int64, device=dev)
    bits[r, i] = s["masks"] if s["tree"] else torch.zeros_like(i)
    by_tree = (bits[:, :, None] >> back.clamp(0, 63)[:, None, :]) & 1 == 1
    by_place = back[:, None, :] <= torch.arange(n, device=dev)[None, :, None]
    seen = (back < 0)[:, None, :] | ((back >= 0)[:, None, :] & (by_tree if s["tree"] else by_place))
    seen = seen & (j < lens[:, None])[:, None, :]
    mine = torch.zeros((R, n), dtype=torch.int64, device=dev)
    mine[r, i] = s["positions"].long()
    theirs = torch.where(back < 0, j[None, :], mine.gather(1, back.clamp(0, n - 1)))
    frozen = torch.tensor(s["mask"], dtype=torch.bool, device=dev)
    if any(s["mask"]):
        d = (mine[:, :, None] - theirs[:, None, :]).clamp(0, L - 1)
        some = frozen.nonzero()[:, 0]
        fixed = s["alpha"][some][:, theirs.clamp(0, L - 1)].permute(1, 0, 2)[:, None] + s["rho"][some][:, d].permute(1, 2, 0, 3)
        scores[:, :, some] = fixed
    scores = torch.where(seen[:, :, None, :], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total == 0, 1.0, total)).view(R, n, H // g, g, L).permute(0, 2, 1, 3, 4).reshape(R, H // g, n * g, L)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)).view(R, H // g, n, g, D).permute(0, 2, 1, 3, 4).reshape(R, n, H, D)
    lse = torch.where(frozen, 0.0, (top + total.log())[..., 0])
    return {"O": s["O"].copy_(o[r, i]), "LSE": s["LSE"].copy_(lse[r, i])}


# --------------------------------------------------------------------------------------------------- the framework's calls
@functools.lru_cache(maxsize=None)
def _context(device):
    import paper_2609_34650_b200 as saf
    return saf.Context(device)                             # one a process, as a program keeps it


def _problem(s):
    """The description of a case's tensors, which a program makes once for its shapes."""
    if "problem" not in s:
        import paper_2609_34650_b200 as saf
        if s["op"] == ROTARY:
            fwd = saf.make_rotary(s["q"], s["k"], s["q_out"], s["k_out"], s["rot"], s["interleaved"], s["mscale"])
            bwd = saf.make_rotary(s["dq"], s["dk"], s["dq_out"], s["dk_out"], s["rot"], s["interleaved"], s["mscale"]) if s["back"] else None
            s["problem"] = (fwd, bwd)
        elif s["op"] == PLAN:
            s["problem"] = saf.make_cache(s["R"], s["N"], s["page"], s["pages"], s["max_pages"])
        else:
            sizes = (s["R"], s["N"], s["page"], s["pages"], s["max_pages"])
            caches = {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
            if s["op"] == APPEND:
                s["problem"] = (saf.make_cache(*sizes, **caches, v_like=s["v"]),
                                saf.make_rotary(s["q"], s["k"], s["q_out"], None, s["rot"], s["interleaved"], s["mscale"]))
            else:
                s["problem"] = saf.make_cache(*sizes, **caches, q_like=s["q"], o_like=s["O"], Tp=s["max_len"], max_len=s["max_len"],
                                              max_new=s["max_new"])
    return s["problem"]


def _own_plan(s, ctx):
    out = s["out"]
    ctx.saf_cache_plan(_problem(s), s["ctx"], s["new"], s.get("parents"), s["held"], out["held"], s["count"], out["count"], s["free"],
                       s["table"], out["offsets"], out["kv_lens"], out["slots"], out["positions"], out.get("masks"), out["missing"])
    return {**out, "table": s["table"], "free": s["free"]}


def _own_rotary(s, ctx):
    fwd, bwd = _problem(s)
    ctx.saf_rotary_fwd(fwd, s["q"], s["k"], s["positions"], s["freqs"], s["q_out"], s["k_out"])
    out = {"q": s["q_out"], "k": s["k_out"]}
    if s["back"]:
        ctx.saf_rotary_bwd(bwd, s["dq"], s["dk"], s["positions"], s["freqs"], s["dq_out"], s["dk_out"])
        out["dq"], out["dk"] = s["dq_out"], s["dk_out"]
    return out


def _own_append(s, ctx):
    c, r = _problem(s)
    ctx.saf_cache_append(c, r, s["q"], s["k"], s["v"], s["slots"], s["positions"], s["freqs"], s["q_out"], s["k_cache"], s["v_cache"])
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attend(s, ctx):
    ctx.saf_cache_attn(_problem(s), s["q"], s["k_cache"], s["v_cache"], s["table"], s["offsets"], s["kv_lens"], s["positions"], s["masks"],
                       s["mask"], s["alpha"], s["rho"], s["O"], s["LSE"])
    return {"O": s["O"], "LSE": s["LSE"]}


def run(state):
    op = state["op"]
    if own:
        ctx = _context(torch.cuda.current_device())
        return {PLAN: _own_plan, ROTARY: _own_rotary, APPEND: _own_append, ATTEND: _own_attend}[op](state, ctx)
    return {PLAN: _plain_plan, ROTARY: _plain_rotary, APPEND: _plain_append, ATTEND: _plain_attend}[op](state)


# --------------------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == ROTARY:
        q, k = case["B"] * case["H"] * case["T"] * case["D"], case["B"] * (case["H"] // case["group"]) * case["T"] * case["D"]
        bytes_ = 4 * (q + k) + 4 * case["B"] * case["T"]
        flops = 3 * (q + k) * case["rot"] // case["D"]
        if case["back"]:
            bytes_ += (q + k) * ((4 if case["grads"] == "fp32" else 2) + (4 if case["out"] == "fp32" else 2))
            flops *= 2
        return {"bytes": bytes_, "flops": flops}
    ctx, many = _lengths(case)
    tokens = sum(many)
    if case["op"] == PLAN:
        # lengths and held pages in, their successors out, new pages from stack to table, three words a token (and a set of 64
        # bits and a parent in a tree), one table entry a page that new tokens touch
        page = case["page"]
        fresh = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(ctx, many))
        return {"bytes": 4 * (7 * case["R"] + 2 * fresh + 2 * tokens) + (12 * tokens if case["tree"] else 0), "flops": 0}
    H, g, D = case["H"], case["group"], case["D"]
    if case["op"] == APPEND:
        rows = tokens * (H + 2 * (H // g)) * D
        return {"bytes": 4 * rows + 8 * tokens, "flops": 3 * tokens * (H + H // g) * case["rot"]}
    mask = _frozen(case)
    keys = sum(c + n for c, n in zip(ctx, many))
    with_k = sum(1 for a in range(H // g) if not all(mask[a * g:(a + 1) * g]))      # heads whose keys are read at all
    ordinary = H - sum(mask)
    pairs = sum((c + (n + 1) / 2) * n for c, n in zip(ctx, many))
    bytes_ = 2 * keys * D * (with_k + H // g) + tokens * D * (2 * ordinary + (4 if case["out"] == "fp32" else 2) * H) + 4 * tokens * H
    bytes_ += 8 * sum(mask) * max(ctx)
    return {"bytes": int(bytes_), "flops": int(pairs * D * (4 * ordinary + 2 * sum(mask)))}


# --------------------------------------------------------------------------------------------------- in 64 bits
def _exact_turn(x, positions, s, back=False):
    """x [..., T, D] as complex numbers times exp(i angle) (its conjugate on the way back)."""
    x, rot = x.double(), s["rot"]
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if s["interleaved"] else (2, rot // 2))
    pairs = pairs if s["interleaved"] else pairs.transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = positions.double().unsqueeze(-1) * s["freqs"]
    z = z * torch.polar(torch.full_like(angle, s["mscale"]), -angle if back else angle)
    pairs = torch.view_as_real(z)
    pairs = pairs if s["interleaved"] else pairs.transpose(-1, -2)
    return torch.cat([pairs.flatten(-2), x[..., rot:]], -1)


def _exact_attend(s):
    H, g, D, page = s["H"], s["group"], s["D"], s["page"]
    O, LSE = torch.zeros(s["O"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["LSE"].shape, dtype=torch.float64, device="cuda")
    offs, ctx, lens = s["offsets"].tolist(), s["ctx"].tolist(), s["kv_lens"].tolist()
    for r in range(s["R"]):
        a, n, L = offs[r], offs[r + 1] - offs[r], lens[r]
        ids = s["table"][r, :-(-L // page)].long()
        pos = torch.cat([torch.arange(ctx[r], device="cuda"), s["positions"][a:a + n].long()])
        see = torch.ones((n, L), dtype=torch.bool, device="cuda")
        for i in range(n):
            if s["tree"]:
                word = int(s["masks"][a + i])
                see[i, ctx[r]:] = torch.tensor([(word >> j) & 1 == 1 for j in range(n)], device="cuda")
            else:
                see[i, ctx[r] + i + 1:] = False
        for c in range(H // g):
            k = s["k_cache"][ids, c].reshape(-1, D)[:L].double()
            v = s["v_cache"][ids, c].reshape(-1, D)[:L].double()
            for h in range(c * g, c * g + g):
                if s["mask"][h]:
                    d = pos[ctx[r]:, None] - pos[None, :]
                    x = s["alpha"][h].double()[pos][None, :] + s["rho"][h].double()[d.clamp(min=0)]
                else:
                    x = s["q"][a:a + n, h].double() @ k.T / math.sqrt(D)
                x = x.masked_fill(~see, -math.inf)
                O[a:a + n, h] = torch.softmax(x, -1) @ v
                if not s["mask"][h]:
                    LSE[a:a + n, h] = torch.logsumexp(x, -1)
    return {"O": O, "LSE": LSE}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == PLAN:
        return None                                        # whole numbers throughout
    if case["op"] == ATTEND:
        return _exact_attend(s)
    if case["op"] == ROTARY:
        at = s["positions"][:, None]
        out = {"q": _exact_turn(s["q"], at, s), "k": _exact_turn(s["k"], at, s)}
        if s["back"]:
            out["dq"], out["dk"] = _exact_turn(s["dq"], at, s, back=True), _exact_turn(s["dk"], at, s, back=True)
        return out
    at = s["positions"][None]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    slots = s["slots"].long()
    kc.transpose(1, 2)[slots // s["page"], slots % s["page"]] = _exact_turn(s["k"].transpose(0, 1), at, s).transpose(0, 1)
    vc.transpose(1, 2)[slots // s["page"], slots % s["page"]] = s["v"].double()
    return {"q": _exact_turn(s["q"].transpose(0, 1), at, s).transpose(0, 1), "k_cache": kc, "v_cache": vc}
