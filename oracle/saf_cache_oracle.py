"""Dense fp64 statements of rotary positions and of a step on a paged key/value cache, in plain numpy loops.  Shares no code with the
kernels."""
import math

import numpy as np


def rotary(x, positions, freqs, interleaved=False, mscale=1.0, backward=False):
    """x [B,H,T,D], positions [B,T], freqs [rot/2] (radians per position): pair i of the first rot features turned by position * freq."""
    y = np.array(x, dtype=np.float64)
    rot = 2 * len(freqs)
    sign = -1.0 if backward else 1.0
    for i, f in enumerate(freqs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        t = positions.astype(np.float64)[:, None, :] * f
        c, s = mscale * np.cos(t), sign * mscale * np.sin(t)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, trained_len=0):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = 1.0 / base ** (2 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "ramp":
            where = lambda turns: rot * math.log(trained_len / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(math.floor(where(32)), 0), min(math.ceil(where(1)), rot - 1)
            slow = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = slow * f / factor + (1 - slow) * f
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0


def ancestors(parents):
    """Sets (as integers) and depths of one request's drafted tokens."""
    sets, depth = [], []
    for i, p in enumerate(parents):
        p = p if 0 <= p < i else -1
        sets.append((1 << i) | (sets[p] if p >= 0 else 0))
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth


def plan(ctx_lens, new_lens, parents, held, free, table, page, max_pages, N):
    """One step, request after request.  `free`: list, top last; `table`: [R][max_pages].  Returns a dict; inputs are not changed."""
    R = len(ctx_lens)
    held, free, table = list(held), list(free), np.array(table)
    new_held, kv, missing, offsets = list(held), [0] * R, [0] * R, [0]
    slots, positions, masks = np.full(N, -1, np.int32), np.zeros(N, np.int32), np.zeros(N, np.uint64)
    need, end = [], 0
    for r in range(R):
        n = max(new_lens[r], 0)
        end += n
        offsets.append(min(end, N))
        pages = -(-(max(ctx_lens[r], 0) + n) // page)
        refused = ctx_lens[r] < 0 or new_lens[r] < 0 or pages > max_pages or (end > N and n > 0) or (parents is not None and n > 64)
        need.append(None if refused else pages)
    for r in range(R):
        if need[r] is not None and need[r] < held[r]:
            free += [int(x) for x in table[r, need[r]:held[r]]]
            new_held[r] = need[r]
    out_of_pages = False
    for r in range(R):
        if need[r] is None:
            missing[r] = -1
            continue
        grow = max(need[r] - held[r], 0)
        if grow and (out_of_pages or grow > len(free)):
            out_of_pages = True
            missing[r] = grow
            continue
        for col in range(held[r], need[r]):
            table[r, col] = free.pop()
        new_held[r] = need[r]
        kv[r] = ctx_lens[r] + new_lens[r]
    for r in range(R):
        first, n = offsets[r], offsets[r + 1] - offsets[r]
        ctx = max(ctx_lens[r], 0)
        for i in range(n):
            positions[first + i] = ctx + (i if parents is None else 0)
            if need[r] is not None and missing[r] == 0:
                slots[first + i] = table[r, (ctx + i) // page] * page + (ctx + i) % page
        if parents is not None and new_lens[r] <= 64:
            sets, depth = ancestors([int(x) for x in parents[first:first + n]])
            for i in range(n):
                masks[first + i] = sets[i]
                positions[first + i] = ctx + depth[i]
    return {"held": new_held, "free": free, "table": table, "offsets": offsets, "kv_lens": kv, "missing": missing, "slots": slots,
            "positions": positions, "masks": masks}


def attend(q, k, v, ctx, frozen, alpha, rho, positions=None, masks=None, scale=None):
    """One request: q [n,H,D], k and v [len,Hkv,D] (new tokens' included), new token i at place ctx + i.  Returns O [n,H,D], LSE [n,H]
    and, for error bounds, sum of weights times |v| [n,H,D] and the largest sum of |q k| scale [n,H]."""
    n, H, D = q.shape
    g = H // k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    O, A = np.zeros((n, H, D)), np.zeros((n, H, D))
    LSE, S = np.zeros((n, H)), np.zeros((n, H))
    pos = np.concatenate([np.arange(max(ctx, 0)), ctx + np.arange(n) if positions is None else positions]).astype(int)
    for i in range(n):
        own = np.arange(n) <= i if masks is None else np.array([(int(masks[i]) >> j) & 1 == 1 for j in range(n)], dtype=bool)
        seen = np.concatenate([np.ones(max(ctx, 0), bool), own])
        for h in range(H):
            at = np.nonzero(seen & (pos <= pos[max(ctx, 0) + i]) if frozen[h] else seen)[0]
            if len(at) == 0:
                LSE[i, h] = 0.0 if frozen[h] else -np.inf
                continue
            if frozen[h]:
                s = alpha[h, pos[at]].astype(np.float64) + rho[h, pos[max(ctx, 0) + i] - pos[at]]
                S[i, h] = np.abs(s[np.isfinite(s)]).max(initial=0.0)
            else:
                s = k[at, h // g] @ q[i, h] * scale
                S[i, h] = (np.abs(k[at, h // g]) @ np.abs(q[i, h]) * scale).max()
            top = s.max()
            w = np.exp(s - top)
            LSE[i, h] = 0.0 if frozen[h] else top + math.log(w.sum())
            O[i, h] = (w / w.sum()) @ v[at, h // g]
            A[i, h] = (w / w.sum()) @ np.abs(v[at, h // g])
    return O, LSE, A, S
