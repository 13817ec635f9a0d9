"""GPU parity of the norm over all gradients and of clipping against the CPU oracle.

u = 2^-24.  Sums are fp64: the norm is right but for its rounding to fp32 (u, 1e-12 for the sum).  A scaled value carries the factor's rounding, the product's and the
rounding to its type.
"""
import math

import numpy as np
import pytest

from oracle import grads as ogr

pytestmark = pytest.mark.gpu

from gpu_util import host, torch_mod  # noqa: E402

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
SENTINEL = 768.0


@pytest.fixture(scope="module")
def hap():
    import paper_2401_05965_amd as h
    return h


def make(shapes, seed=0, sigma=1.0):
    """shapes: (rows, cols, ld, dtype, shift).  Views into one buffer each; what lies around the values is NaN."""
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    vals, views, whole = [], [], []
    for r, c, ld, dt, shift in shapes:
        td = {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
        buf = torch.full((shift + max(r, 1) * ld + 9,), float("nan"), dtype=td, device="cuda")
        v = buf[shift:shift + r * ld].view(r, ld)[:, :c]
        v.copy_(torch.from_numpy(rng.normal(size=(r, c)) * sigma).to(td))
        vals.append(v.double().cpu().numpy()); views.append(v); whole.append(buf)
    return vals, views, whole


def desc_of(hap, shapes, max_norm):
    return hap.GradDesc([(r, c, ld, hap.BF16 if dt == "bf16" else hap.F32) for r, c, ld, dt, _ in shapes], max_norm)


def run_clip(hap, shapes, max_norm, in_place, seed=0, sigma=1.0):
    torch = torch_mod()
    vals, g, whole = make(shapes, seed, sigma)
    d = desc_of(hap, shapes, max_norm)
    ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda").fill_(255)
    total = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda"); norm = torch.full((1,), float("nan"), device="cuda")
    hap.hap_grad_sumsq(d, g, total, ws)
    want = ogr.sumsq(vals)
    assert float(total) == pytest.approx(want, rel=1e-12, abs=0)
    if in_place:
        outs, around = g, whole
        hap.hap_grad_clip(d, g, g, total, norm)
    else:
        _, outs, around = make([(r, c, ld + 3, dt, (s + 1) % 8) for r, c, ld, dt, s in shapes], seed + 1)
        hap.hap_grad_clip(d, g, outs, total, norm, ldo=[ld + 3 for _, _, ld, _, _ in shapes])
    ref, n = ogr.clip(vals, max_norm, want)
    assert abs(float(norm) - n) <= 1.01 * U * n
    for (r, c, ld, dt, s), o, b, w in zip(shapes, outs, ref, around):
        err = np.abs(host(o) - b)
        exact = n <= max_norm
        assert (err <= (0 if exact else 1.01 * (HALF[dt] + 2 * U)) * np.abs(b) + 2.0 ** -133).all()
        left = torch.ones(w.shape, dtype=torch.bool, device="cuda")
        shift = s if in_place else (s + 1) % 8
        p = ld if in_place else ld + 3
        left[shift:shift + r * p].view(r, p)[:, :c] = False
        assert torch.isnan(w[left]).all(), "written outside of the tensor"


SHAPES = {
    "one": [(1, 1, 1, "f32", 0)],
    "vector": [(1, 1000, 1000, "bf16", 0)],
    "mixed": [(3, 5, 5, "f32", 0), (1, 77, 80, "bf16", 3), (64, 33, 40, "bf16", 0), (0, 9, 9, "f32", 0), (7, 0, 4, "bf16", 0), (130, 64, 64, "bf16", 8), (20, 9000, 9000, "f32", 0)],
    "pitches": [(40, 24, 32, "bf16", 0), (40, 24, 31, "bf16", 0), (33, 1, 64, "f32", 0), (9000, 3, 4, "f32", 1), (5, 8191, 8200, "bf16", 5), (3, 20001, 20008, "f32", 2), (12, 4095, 4096, "bf16", 8)],
    "long": [(1, 8192, 8192, "f32", 0), (1, 8193, 8193, "f32", 1), (1, 3_000_001, 3_000_001, "bf16", 7)],
}


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("in_place", [True, False])
def test_clip_shapes(hap, name, in_place):
    for max_norm in (0.25, 1e9):
        run_clip(hap, SHAPES[name], max_norm, in_place, seed=len(name))


def test_clip_many_tensors(hap):
    """Several tables of arguments, tensors without values among them."""
    shapes = [(i % 5, 1 + (i * 7) % 90, 1 + (i * 7) % 90 + (i % 3), "bf16" if i % 2 else "f32", i % 9) for i in range(333)]
    run_clip(hap, shapes, 1.0, True, seed=3)
    run_clip(hap, shapes, 1.0, False, seed=4)


def test_norms_beyond_the_range_of_fp32_squares(hap):
    for sigma in (1e25, 1e-30):
        run_clip(hap, [(30, 40, 40, "f32", 0), (3, 100, 104, "bf16", 1)], sigma * 3, True, sigma=sigma)


def test_no_tensors(hap):
    torch = torch_mod()
    for shapes in ([], [(0, 5, 5, 0)]):
        d = hap.GradDesc(shapes, 1.0)
        ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda")
        total = torch.full((1,), 5.0, dtype=torch.float64, device="cuda"); norm = torch.full((1,), 5.0, device="cuda")
        hap.hap_grad_sumsq(d, [None] * len(shapes), total, ws)
        hap.hap_grad_clip(d, [None] * len(shapes), [None] * len(shapes), total, norm)
        assert float(total) == 0 and float(norm) == 0


def test_the_devices_norms_add_up(hap):
    """Each device's sum of squares, added up as the All-Reduce does, clips every device's gradients by the norm over all."""
    torch = torch_mod()
    parts = [SHAPES["mixed"], SHAPES["one"], SHAPES["pitches"][:3]]
    total = torch.zeros((1,), dtype=torch.float64, device="cuda")
    made = []
    for i, s in enumerate(parts):
        v, g, _ = make(s, seed=10 + i)
        d = desc_of(hap, s, 0.5)
        ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda"); one = torch.empty_like(total)
        hap.hap_grad_sumsq(d, g, one, ws)
        total += one
        made.append((v, g, d))
    want = ogr.sumsq([x for v, _, _ in made for x in v])
    for v, g, d in made:
        hap.hap_grad_clip(d, g, g, total)
    after = math.sqrt(sum(float((t.double() ** 2).sum()) for _, g, _ in made for t in g))
    assert float(total) == pytest.approx(want, rel=1e-12) and after == pytest.approx(0.5, rel=2.0 ** -8)


def test_norms_that_are_no_numbers(hap):
    """An infinite gradient: factor 0, its own value NaN; a NaN: everything NaN."""
    torch = torch_mod()
    for bad in (float("inf"), float("nan")):
        g = torch.ones(100, device="cuda"); g[7] = bad
        d = hap.GradDesc([(1, 100, 100, hap.F32)], 1.0)
        ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda")
        total = torch.empty((1,), dtype=torch.float64, device="cuda"); norm = torch.empty((1,), device="cuda")
        hap.hap_grad_sumsq(d, [g], total, ws)
        hap.hap_grad_clip(d, [g], [g], total, norm)
        assert torch.isnan(g[7]) and (torch.isnan(g).all() if math.isnan(bad) else ((g == 0).sum() == 99 and float(norm) == bad))


@pytest.mark.parametrize("in_place", [True, False])
def test_factors_below_the_normal_range_of_fp32(hap, in_place):
    """max_norm / norm of 1e-38 and less: the scaled values are ordinary numbers again."""
    for max_norm in (1.0, 1e-3, 1e-6, 1e-12):
        run_clip(hap, [(30, 40, 40, "f32", 0), (3, 100, 104, "bf16", 1), (1, 9, 9, "f32", 1)], max_norm, in_place, sigma=1e36)


def test_a_norm_beyond_fp32_still_scales(hap):
    """The norm itself is +inf in fp32; the factor is taken from the fp64 sum."""
    torch = torch_mod()
    g = torch.full((1 << 12,), 3e38, device="cuda"); g[1::2] = -1e38
    d = hap.GradDesc([(1, 1 << 12, 1 << 12, hap.F32)], 1.0)
    ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda")
    total = torch.empty((1,), dtype=torch.float64, device="cuda"); norm = torch.empty((1,), device="cuda"); out = torch.empty_like(g)
    hap.hap_grad_sumsq(d, [g], total, ws)
    hap.hap_grad_clip(d, [g], [out], total, norm)
    want = g.double() / (g.double() ** 2).sum().sqrt()
    assert float(norm) == math.inf and ((out.double() - want).abs() <= 3.03 * U * want.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_that_the_last_level_cache_does_not_hold(hap, dtype):
    """280 MB of gradients, scaled into other buffers and in place: whole tensors, rows in a pitch, views that begin and end inside a chunk; what lies around them stays."""
    torch = torch_mod()
    td, io, es = {"bf16": (torch.bfloat16, hap.BF16, 2), "f32": (torch.float32, hap.F32, 4)}[dtype]
    gen = torch.Generator(device="cuda"); gen.manual_seed(8)
    n = 280_000_000 // es
    shapes = [(1, n // 2 + 5, n // 2 + 5, 3), (999, 4091, 4096, 0), (n // 2 // 2048, 2048, 2048, 0), (1, 8193, 8193, 7)]
    bufs = [torch.empty((s + r * ld + 11,), dtype=td, device="cuda").normal_(0, 1, generator=gen) for r, _, ld, s in shapes]
    cut = lambda bs: [b[s:s + r * ld].view(r, ld)[:, :c] for b, (r, c, ld, s) in zip(bs, shapes)]
    g = cut(bufs)
    assert sum(t.numel() for t in g) * es > 256 << 20
    d = hap.GradDesc([(r, c, ld, io) for r, c, ld, _ in shapes], 0.75)
    ws = torch.empty((hap.hap_grad_sumsq_workspace(d),), dtype=torch.uint8, device="cuda")
    total, norm = torch.empty((1,), dtype=torch.float64, device="cuda"), torch.empty((1,), device="cuda")
    hap.hap_grad_sumsq(d, g, total, ws)
    want = sum(float((t.double() ** 2).sum()) for t in g)
    assert float(total) == pytest.approx(want, rel=1e-12)
    factor = 0.75 / math.sqrt(want)
    obufs = [torch.full_like(b, SENTINEL) for b in bufs]
    outs = cut(obufs)
    hap.hap_grad_clip(d, g, outs, total, norm)
    assert float(norm) == pytest.approx(math.sqrt(want), rel=1.01 * U)
    for t, o in zip(g, outs):
        ref = t.double() * factor
        assert ((o.double() - ref).abs() <= 1.01 * (HALF[dtype] + 2 * U) * ref.abs()).all()
    for o in outs:
        o.fill_(SENTINEL)
    # nothing outside of the views was written
    assert all((b == SENTINEL).all() for b in obufs)
    hap.hap_grad_clip(d, g, outs, total)
    before = [b.clone() for b in bufs]
    hap.hap_grad_clip(d, g, g, total)
    for a, b in zip(g, outs):
        assert torch.equal(a, b)
    for t, b in zip(cut(before), g):
        t.copy_(b)
    assert all(torch.equal(a, b) for a, b in zip(before, bufs))
