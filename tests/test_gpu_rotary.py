"""Rotary positions on the GPU against the fp64 oracle: layouts, dtypes, parts of a head, far positions, in place, refusals."""
import numpy as np
import pytest
import torch

import paper_2609_34650_b200 as saf
from oracle import saf_cache_oracle as orc

pytestmark = pytest.mark.gpu


def heads(gen, B, H, T, D, layout, dtype):
    if layout == "bhtd":
        return torch.randn((B, H, T, D), generator=gen, device="cuda").to(dtype)
    if layout == "bthd":
        return torch.randn((B, T, H, D), generator=gen, device="cuda").to(dtype).transpose(1, 2)
    return torch.randn((B, T, H + 3, D + 8), generator=gen, device="cuda").to(dtype)[:, :, 1:H + 1, 8:].transpose(1, 2)   # a slice


def bound(x, want, freqs, mscale, out_dtype):
    """Cosine and sine to 2 ulp, the angle's rounding to fp32 half a turn off by at most 2^-25 of a turn, their product with mscale, two
    products and a sum in fp32: 8 * 2^-23 of the pair's two magnitudes; half a step of the output's type."""
    pair = np.abs(x).max() * 2 * max(mscale, 1.0)
    return 8 * 2.0 ** -23 * pair + (torch.finfo(out_dtype).eps / 2) * np.abs(want)


def f64(t):
    return t.double().cpu().numpy()


CASES = [  # B, Hq, Hk, T, D, rot, interleaved, layout, in, out
    (1, 1, 1, 1, 64, 64, False, "bhtd", "bf16", "bf16"),
    (2, 12, 12, 129, 64, 64, False, "bthd", "bf16", "bf16"),
    (2, 12, 3, 129, 64, 64, True, "slice", "bf16", "bf16"),
    (3, 8, 2, 333, 128, 96, True, "bthd", "fp32", "bf16"),
    (1, 5, 5, 77, 96, 48, False, "slice", "bf16", "fp32"),
    (1, 4, 4, 2500, 96, 96, False, "bhtd", "fp32", "fp32"),
    (2, 3, 0, 50, 64, 20, False, "bthd", "bf16", "bf16"),
    (2, 0, 3, 50, 40, 40, True, "bhtd", "bf16", "bf16"),
    (1, 2, 1, 9, 8, 2, True, "bthd", "fp32", "fp32"),
    (1, 2, 2, 9, 512, 512, False, "bthd", "bf16", "bf16"),
    (1, 2, 2, 9, 512, 510, False, "bthd", "bf16", "bf16"),
    (1, 2, 2, 33, 64, 0, False, "bthd", "bf16", "fp32"),
]


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_against_oracle(case, backward, far):
    B, Hq, Hk, T, D, rot, inter, layout, ti, to = case
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}
    gen = torch.Generator(device="cuda").manual_seed(3)
    ctx = saf.Context(0)
    q = heads(gen, B, Hq, T, D, layout, dt[ti]) if Hq else None
    k = heads(gen, B, Hk, T, D, layout, dt[ti]) if Hk else None
    qo, ko = (None if t is None else heads(gen, B, t.shape[1], T, D, layout, dt[to]) for t in (q, k))
    freqs, mscale = saf.saf_rotary_freqs(rot, 10000.0, saf.SAF_ROPE_RAMP, 8.0, 4096) if rot > 2 else (np.full(max(rot // 2, 0), 0.7), 1.0)
    pos = torch.randint(0, 10 ** 7, (B, T), generator=gen, device="cuda").int() if far else None
    prob = saf.make_rotary(q, k, qo, ko, rot, inter, mscale)
    call = ctx.saf_rotary_bwd if backward else ctx.saf_rotary_fwd
    call(prob, q, k, pos, torch.from_numpy(freqs).cuda() if rot else None, qo, ko)
    torch.cuda.synchronize()
    where = pos.cpu().numpy() if far else np.tile(np.arange(T), (B, 1))
    for x, y in ((q, qo), (k, ko)):
        if x is None:
            continue
        want = orc.rotary(f64(x), where, freqs, inter, mscale, backward)
        assert (np.abs(f64(y) - want) <= bound(f64(x), want, freqs, mscale, dt[to])).all()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [64, 20])
def test_in_place(inter, rot):
    gen = torch.Generator(device="cuda").manual_seed(4)
    ctx = saf.Context(0)
    q, k = heads(gen, 2, 4, 65, 64, "bthd", torch.bfloat16), heads(gen, 2, 2, 65, 64, "bthd", torch.bfloat16)
    f = torch.from_numpy(saf.saf_rotary_freqs(rot)[0]).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ctx.saf_rotary_fwd(saf.make_rotary(q, k, qo, ko, rot, inter), q, k, None, f, qo, ko)
    ctx.saf_rotary_fwd(saf.make_rotary(q, k, q, k, rot, inter), q, k, None, f, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_writes_nothing_but_its_output():
    gen = torch.Generator(device="cuda").manual_seed(5)
    ctx = saf.Context(0)
    q = heads(gen, 2, 4, 37, 64, "bthd", torch.bfloat16)
    whole = torch.full((2, 37, 7, 80), 3.0, device="cuda", dtype=torch.bfloat16)
    out = whole[:, :, 1:5, 8:72].transpose(1, 2)
    ctx.saf_rotary_fwd(saf.make_rotary(q, None, out, None, 64), q, None, None, torch.from_numpy(saf.saf_rotary_freqs(64)[0]).cuda(), out, None)
    out.fill_(3.0)
    assert (whole == 3.0).all()


def test_backward_is_the_adjoint_and_matches_differences():
    """<dy, R x> = <R^T dy, x>, and differences of the GPU's own forward in fp32."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    ctx = saf.Context(0)
    x, dy = (heads(gen, 1, 2, 5, 64, "bhtd", torch.float32) for _ in range(2))
    freqs, m = saf.saf_rotary_freqs(48, 10000.0, saf.SAF_ROPE_RAMP, 8.0, 64)
    f = torch.from_numpy(freqs).cuda()
    prob = saf.make_rotary(x, None, x, None, 48, True, m)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    ctx.saf_rotary_bwd(prob, dy, None, None, f, dx, None)

    def value(z):
        ctx.saf_rotary_fwd(prob, z, None, None, f, y, None)
        return float((y.double() * dy.double()).sum())
    a, b = value(x), float((dx.double() * x.double()).sum())
    assert abs(a - b) <= 8 * 2.0 ** -23 * 2 * m * float((x.abs().double() + 4).mul(dy.abs().double() + 4).sum())
    for at in ((0, 0, 3, 0), (0, 1, 4, 47), (0, 1, 2, 63), (0, 0, 0, 5)):
        hi, lo = x.clone(), x.clone()
        hi[at] += 1.0
        lo[at] -= 1.0                                       # the map is linear: a step of one is as good as any
        # two values of at most 640 products, each off by 8 * 2^-23 of its pair
        assert abs((value(hi) - value(lo)) / 2 - float(dx[at])) <= 1e-3


def test_no_rotation_of_an_empty_call():
    ctx = saf.Context(0)
    p = saf.SafRotary()
    p.B = p.T = 1
    p.D, p.rot_dim = 64, 64
    ctx.saf_rotary_fwd(p, None, None, None, None, None, None)


def test_refusals():
    gen = torch.Generator(device="cuda").manual_seed(7)
    ctx = saf.Context(0)
    q, k = heads(gen, 2, 4, 16, 64, "bthd", torch.bfloat16), heads(gen, 2, 2, 16, 64, "bthd", torch.bfloat16)
    f = torch.from_numpy(saf.saf_rotary_freqs(64)[0]).cuda()
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 5.0)

    def refused(code, change=None, **args):
        p = saf.make_rotary(q, k, qo, ko, 64)
        if change:
            change(p)
        a = {"q": q, "k": k, "f": f, "qo": qo, "ko": ko, **args}
        for call in (ctx.saf_rotary_fwd, ctx.saf_rotary_bwd):
            with pytest.raises(saf.SafError) as e:
                call(p, a["q"], a["k"], None, a["f"], a["qo"], a["ko"])
            assert e.value.code == code

    for name, value, code in (("B", 0, 1), ("T", 0, 1), ("Hq", -1, 1), ("Hk", 70000, 1), ("D", 0, 1), ("D", 68, 2), ("D", 520, 2), ("rot_dim", 66, 1),
                              ("rot_dim", 63, 1), ("rot_dim", -2, 1), ("in_dtype", 2, 2), ("out_dtype", -1, 2), ("B", 1 << 30, 1)):
        refused(code, lambda p: setattr(p, name, value))
    for name in ("q_strides", "k_strides", "qo_strides", "ko_strides"):
        for i in range(3):
            refused(1, lambda p: getattr(p, name).__setitem__(i, 12))
            refused(1, lambda p: getattr(p, name).__setitem__(i, -64))
    for name in ("q", "k", "f", "qo", "ko"):
        refused(1, **{name: None})
    for name, t in (("q", q), ("k", k), ("qo", qo), ("ko", ko)):
        refused(1, **{name: t.flatten()[1:]})
    torch.cuda.synchronize()
    assert (qo == 5.0).all() and (ko == 5.0).all()


def test_around_the_layer():
    """Rotation, layer, layer's backward, rotation's backward: the update of a layer with rotary positions against the oracles."""
    from oracle import saf_oracle as layer
    from gpu_util import assert_close
    gen = torch.Generator(device="cuda").manual_seed(8)
    ctx = saf.Context(0)
    B, H, T, D = 1, 4, 200, 64
    mask = np.array([0, 1, 0, 0], np.uint8)
    q, k, v, do = (heads(gen, B, H, T, D, "bthd", torch.bfloat16) for _ in range(4))
    alpha = torch.randn((H, T), generator=gen, device="cuda")
    rho = -0.05 * torch.arange(T, device="cuda").float() + 0.1 * torch.randn((H, T), generator=gen, device="cuda")
    logz = torch.zeros_like(alpha)
    freqs, _ = saf.saf_rotary_freqs(64)
    f = torch.from_numpy(freqs).cuda()
    qr, kr, O = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    lse = torch.empty((B, H, T), device="cuda")
    dqr, dkr, dv = (torch.empty((B, H, T, D), device="cuda") for _ in range(3))
    dq, dk = torch.empty_like(q, dtype=torch.float32), torch.empty_like(k, dtype=torch.float32)
    prob = saf.make_problem(qr, T, k_like=kr, v_like=v, o_like=O)
    ctx.saf_pattern_prepare(mask, alpha, rho, logz)
    ctx.saf_rotary_fwd(saf.make_rotary(q, k, qr, kr, 64), q, k, None, f, qr, kr)
    ctx.saf_hybrid_attn_fwd(prob, qr, kr, v, mask, alpha, rho, logz, O, lse)
    ctx.saf_hybrid_attn_bwd(prob, qr, kr, v, O, do, lse, mask, alpha, rho, logz, dqr, dkr, dv)
    ctx.saf_rotary_bwd(saf.make_rotary(dqr, dkr, dq, dk, 64), dqr, dkr, None, f, dq, dk)
    torch.cuda.synchronize()
    assert ctx.saf_last_device_status()[0] == saf.SAF_OK
    pos = np.arange(T)[None]
    # (the layer is fed what the rotation rounded to bf16)
    eo, _ = layer.hybrid_attn_fwd(f64(qr), f64(kr), f64(v), mask, f64(alpha), f64(rho))
    eq, ek, ev = layer.hybrid_attn_bwd(f64(qr), f64(kr), f64(v), f64(do), mask, f64(alpha), f64(rho))
    assert_close(f64(O), eo, "O")
    assert_close(f64(dq), orc.rotary(eq, pos, freqs, backward=True), "dQ")
    assert_close(f64(dk), orc.rotary(ek, pos, freqs, backward=True), "dK")
    assert_close(f64(dv), ev, "dV")
