"""CPU checks of the oracle of rotary positions and the paged cache, of the host-only frequencies and of the structs' layouts."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2609_34650_b200 as saf
from oracle import saf_cache_oracle as orc
from oracle import saf_oracle as layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_34650_b200.build import build_library
    build_library()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_scores_depend_on_distance_alone(interleaved):
    rng = np.random.default_rng(0)
    f, _ = orc.frequencies(16)
    q, k = rng.standard_normal((2, 1, 1, 1, 24))
    score = lambda a, b: (orc.rotary(q, np.array([[a]]), f, interleaved) * orc.rotary(k, np.array([[b]]), f, interleaved)).sum()  # noqa: E731
    assert abs(score(100, 93) - score(1007, 1000)) < 1e-10
    assert abs(score(100, 93) - score(100, 94)) > 1e-6
    assert np.allclose(orc.rotary(q, np.array([[0]]), f, interleaved), q)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_backward_is_the_gradient(interleaved):
    rng = np.random.default_rng(1)
    f, m = orc.frequencies(8, scaling="ramp", factor=4.0, trained_len=128)
    x, dy = rng.standard_normal((2, 1, 2, 3, 12))
    pos = np.array([[5, 0, 77]])
    dx = orc.rotary(dy, pos, f, interleaved, m, backward=True)
    for at in np.ndindex(x.shape):
        step = np.zeros_like(x)
        step[at] = 1e-6
        diff = ((orc.rotary(x + step, pos, f, interleaved, m) - orc.rotary(x - step, pos, f, interleaved, m)) * dy).sum() / 2e-6
        assert abs(diff - dx[at]) < 1e-8


@pytest.mark.parametrize("scaling,factor,trained", [("plain", 1.0, 0), ("linear", 4.0, 0), ("base", 8.0, 0), ("ramp", 8.0, 4096), ("ramp", 1.0, 32)])
@pytest.mark.parametrize("rot", [2, 6, 64, 128])
def test_frequencies(scaling, factor, trained, rot):
    kind = {"plain": saf.SAF_ROPE_PLAIN, "linear": saf.SAF_ROPE_LINEAR, "base": saf.SAF_ROPE_BASE, "ramp": saf.SAF_ROPE_RAMP}[scaling]
    if scaling == "base" and rot == 2:
        with pytest.raises(saf.SafError):
            saf.saf_rotary_freqs(rot, 10000.0, kind, factor, trained)
        return
    got, m = saf.saf_rotary_freqs(rot, 10000.0, kind, factor, trained)
    want, wm = orc.frequencies(rot, 10000.0, scaling, factor, trained)
    assert np.allclose(got, want, rtol=1e-13, atol=0) and abs(m - wm) < 1e-7


@pytest.mark.parametrize("rot,base,kind,factor,trained", [(0, 1e4, 0, 1.0, 0), (3, 1e4, 0, 1.0, 0), (8, 1.0, 0, 1.0, 0), (8, 1e4, 4, 1.0, 0), (8, 1e4, -1, 1.0, 0),
                                                          (8, 1e4, 1, 0.5, 0), (8, 1e4, 3, 2.0, 0), (8, float("nan"), 0, 1.0, 0), (8, 1e4, 1, float("inf"), 0)])
def test_frequencies_refuse(rot, base, kind, factor, trained):
    with pytest.raises(saf.SafError) as e:
        saf.saf_rotary_freqs(rot, base, kind, factor, trained)
    assert e.value.code == 1


def test_plan_gives_back_before_it_takes_and_stops_at_the_first_that_finds_too_few():
    table = np.array([[7, 8, 9], [1, 0, 0], [2, 0, 0], [0, 0, 0]])
    #        gives back two, wants one, wants two (too few are left), wants none
    got = orc.plan([3, 4, 1, 0], [1, 1, 8, 0], None, [3, 1, 1, 0], [5], table, 4, 3, 12)
    assert got["missing"] == [0, 0, 0, 0] and got["table"][1, 1] == 9 and list(got["table"][2, 1:]) == [8, 5] and got["free"] == []
    got = orc.plan([3, 4, 1, 0], [1, 1, 8, 0], None, [1, 1, 1, 0], [5], table, 4, 3, 12)
    assert got["missing"] == [0, 0, 2, 0] and got["kv_lens"] == [4, 5, 0, 0] and got["free"] == []
    assert list(got["slots"][2:10]) == [-1] * 8


def test_ancestors_of_a_tree():
    sets, depth = orc.ancestors([-1, 0, 0, 2, -1, 4, 9, -5])
    assert sets == [1, 3, 5, 13, 16, 48, 64, 128] and depth == [0, 1, 1, 2, 0, 1, 0, 0]


def test_cached_steps_equal_the_layer():
    """Token by token over the cache, and a tree's paths one by one, give the rows of the square causal layer."""
    rng = np.random.default_rng(2)
    T, H, D = 9, 3, 8
    q, k, v = rng.standard_normal((3, 1, H, T, D))
    mask = np.array([0, 1, 0], np.uint8)
    alpha, rho = rng.standard_normal((2, H, T)).astype(np.float32)
    want, lse = layer.hybrid_attn_fwd(q, k, v, mask, alpha, rho)
    rows = lambda x: x[0].transpose(1, 0, 2)  # noqa: E731
    for t in range(T):
        O, L, _, _ = orc.attend(rows(q)[t:t + 1], rows(k)[:t + 1], rows(v)[:t + 1], t, mask, alpha, rho)
        assert np.allclose(O[0], want[0, :, t], atol=1e-12)
        assert np.allclose(L[0, [0, 2]], lse[0, [0, 2], t], atol=1e-12)
    # two branches from the fifth token: 5 6 7 and a copy of them behind, the copies being other tokens
    sets, depth = orc.ancestors([-1, 0, 1, -1, 3])
    order = [5, 6, 7, 5, 6]
    kk = np.concatenate([rows(k)[:5], rows(k)[order]])
    vv = np.concatenate([rows(v)[:5], rows(v)[order]])
    O, _, _, _ = orc.attend(rows(q)[order], kk, vv, 5, mask, alpha, rho, positions=5 + np.array(depth), masks=sets)
    for i, t in enumerate(order):
        assert np.allclose(O[i], want[0, :, t], atol=1e-12)


@pytest.mark.parametrize("name,cls,words", [("saf_rotary", "SafRotary", 10), ("saf_cache", "SafCache", 14)])
def test_struct_layout_matches_header(tmp_path, name, cls, words):
    cls = getattr(saf, cls)
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    fields = [f for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "saf.h"\nint main(void) {\n'
                   f'  printf("%zu\\n", sizeof({name}));\n' + "".join(f'  printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields)
                   + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]
    assert getattr(cls, "q_strides").offset == 4 * words


def test_make_cache_refuses_arrays_that_do_not_fit_together():
    torch = pytest.importorskip("torch")
    kc = torch.zeros((5, 3, 16, 64), dtype=torch.bfloat16)
    q = torch.zeros((7, 6, 64), dtype=torch.bfloat16)
    c = saf.make_cache(2, 7, 16, 5, 4, k_cache=kc, v_cache=kc, q_like=q, o_like=q, v_like=q[:, :3])
    assert (c.H, c.kv_group, c.D, c.o_dtype) == (6, 2, 64, 0)
    for change in (dict(q_like=q[:, :4]), dict(o_like=q[:, :3]), dict(v_like=q), dict(v_cache=kc[:, :2]), dict(k_cache=kc[:4]), dict(q_like=q[:5])):
        with pytest.raises(AssertionError):
            saf.make_cache(2, 7, 16, 5, 4, **dict(dict(k_cache=kc, v_cache=kc, q_like=q, o_like=q, v_like=q[:, :3]), **change))


def test_make_rotary_refuses_arrays_that_do_not_fit_together():
    torch = pytest.importorskip("torch")
    q, k = torch.zeros((2, 4, 9, 64)), torch.zeros((2, 2, 9, 64))
    r = saf.make_rotary(q, k, q, k, 64)
    assert (r.B, r.T, r.Hq, r.Hk, r.D) == (2, 9, 4, 2, 64)
    for args in ((q, k[:, :, :8], q, k[:, :, :8]), (q, k[:1], q, k[:1]), (q, k, q[:, :3], k), (q, k, q, k.bfloat16()), (q, k[0], q, k[0])):
        with pytest.raises(AssertionError):
            saf.make_rotary(*args, 64)
