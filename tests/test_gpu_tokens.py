"""GPU parity of the tokens' way to the experts and back (plan, dispatch, combine and their gradients) against the CPU oracle.

Positions, counts and moved rows are compared exactly.  u = 2^-24: a sum over k choices is off by at most (k + 1) u of its terms' magnitudes, a scalar product over h values (h / 64 + 8
additions on the way of a term, one rounding of its product) by (h / 64 + 9) u, and what is stored in the type by half a step of it.
"""
import numpy as np
import pytest

from oracle import routing as ort

pytestmark = pytest.mark.gpu

from gpu_util import host, torch_mod  # noqa: E402

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
SENTINEL = 768.0


@pytest.fixture(scope="module")
def hap():
    import paper_2401_05965_amd as h
    return h


def run_plan(hap, idx, E, C):
    torch = torch_mod()
    T, k = idx.shape
    d = torch.from_numpy(idx.astype(np.int32)).cuda()
    pos = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    rows = torch.full((E,), -9, dtype=torch.int32, device="cuda"); counts = torch.full_like(rows, -9)
    ws = torch.empty((max(hap.hap_moe_plan_workspace(T, k, E), 16),), dtype=torch.uint8, device="cuda").fill_(255)
    hap.hap_moe_plan(T, k, E, C, d, pos, rows, counts, ws)
    return d, pos, rows, counts


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 64), (7, 3, 5), (64, 1, 2), (65, 2, 30), (500, 8, 256), (1025, 7, 1024), (4096, 2, 8), (8192, 1, 3), (8193, 1, 3), (9001, 3, 30), (30011, 8, 1000),
                                   (200003, 3, 17), (32768, 1, 30), (10923, 3, 30), (349526, 3, 1000), (1300001, 1, 5)])
def test_plan(hap, T, k, E):
    """One workgroup and many; a popular expert, absent ones, choices that are no experts; capacities of 0, some and plenty."""
    rng = np.random.default_rng(T + E)
    idx = rng.integers(0, E, (T, k))
    idx[rng.random(idx.shape) < 0.4] = E // 2
    bad = rng.random(idx.shape) < 0.1
    idx[bad] = rng.choice([-1, E, 2 ** 31 - 1, -2 ** 31], bad.sum())
    flat = idx.reshape(-1)
    valid = (flat >= 0) & (flat < E)
    counts_o = np.bincount(flat[valid], minlength=E)
    order = np.argsort(np.where(valid, flat, E), kind="stable")
    place = np.empty(flat.size, dtype=np.int64)
    start = np.concatenate([[0], np.cumsum(counts_o)])
    place[order[:valid.sum()]] = np.arange(valid.sum()) - start[flat[order[:valid.sum()]]]
    for C in (0, max(1, int(counts_o.mean() * 0.7)), T * k + 1):
        _, pos, rows, counts = run_plan(hap, idx, E, C)
        want = np.where(valid & (place < C), place, -1).reshape(T, k)
        if T * k <= 4000:
            po, ro, co = ort.plan(idx, E, C)
            assert (want == po).all() and (np.minimum(counts_o, C) == ro).all() and (counts_o == co).all()
        assert (pos.cpu().numpy() == want).all() and (counts.cpu().numpy() == counts_o).all() and (rows.cpu().numpy() == np.minimum(counts_o, C)).all()


def test_plan_of_no_tokens_and_without_counts(hap):
    torch = torch_mod()
    rows = torch.full((9,), -9, dtype=torch.int32, device="cuda")
    hap.hap_moe_plan(0, 2, 9, 5, None, None, rows)
    assert (rows.cpu() == 0).all()
    idx = torch.zeros((3, 1), dtype=torch.int32, device="cuda"); pos = torch.empty_like(idx)
    hap.hap_moe_plan(3, 1, 9, 2, idx, pos, rows)
    assert pos.cpu().flatten().tolist() == [0, 1, -1] and rows.cpu().tolist() == [2] + [0] * 8


def placed(values, dtype, ld, shift=0):
    """[..., rows, n] float64 -> (values as stored, device view with pitch ld); the pitch's gaps hold the sentinel."""
    torch = torch_mod()
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    n = values.shape[-1]
    R = int(np.prod(values.shape[:-1]))
    buf = torch.full((R * ld + shift,), SENTINEL, dtype=td, device="cuda")
    view = buf[shift:].view(*values.shape[:-1], ld)
    view[..., :n] = torch.from_numpy(values).to(td).cuda()
    return view[..., :n].double().cpu().numpy(), view


def run_tokens(hap, dtype, T, k, E, C, h, offs, full, pt=0, pe=0, shift=0, seed=0):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    idx = np.argsort(rng.random((T, max(E, k))), axis=1)[:, :k] if E >= k else rng.integers(0, E, (T, k))
    idx = np.where(rng.random(idx.shape) < 0.1, -1, idx)
    if T > 2:
        idx[1] = -1                                       # a token that goes nowhere
        idx[2] = idx[2, 0]                                # one expert k times
    di, pos, rows, _ = run_plan(hap, idx, E, C)
    p = pos.cpu().numpy()
    ldt, lde = h + pt, h + pe
    live = np.arange(C)[None, :] < rows.cpu().numpy()[:, None]
    poison = lambda v: np.where(live[:, :, None], v, np.nan)
    xh, x = placed(rng.normal(size=(T, h)), dtype, ldt, shift)
    Yh, Y = placed(poison(rng.normal(size=(E, C, h))), dtype, lde, shift)
    gh, g = placed(rng.normal(size=(T, h)), dtype, ldt, shift)
    dXh, dX = placed(poison(rng.normal(size=(E, C, h))), dtype, lde, shift)
    w = rng.normal(size=(T, k)).astype(np.float32)
    wn = np.where(p < 0, np.nan, w).astype(np.float32)     # weights of dropped choices are not looked at
    wd = torch.from_numpy(wn).cuda()
    for j in range(len(offs) - 1):
        lo, hi = offs[j], offs[j + 1]
        part = slice(0, E) if full else slice(lo, hi)
        shape = (E if full else hi - lo, C, h)
        blank = lambda s, ld: placed(np.full(s, SENTINEL), dtype, ld, shift)[1]
        Xd, dYd, outd, dxd = blank(shape, lde), blank(shape, lde), blank((T, h), ldt), blank((T, h), ldt)
        dwd = torch.full((T, k), float("nan"), device="cuda")
        d = hap.MoeTokensDesc(T, k, E, C, h, offs, hap.BF16 if dtype == "bf16" else hap.F32, ldt, lde, operands_are_full=full)
        Yj, dXj = Y[part], dX[part]
        hap.hap_moe_dispatch_fwd(d, j, x, di, pos, Xd)
        hap.hap_moe_combine_fwd(d, j, Yj, di, pos, wd, outd)
        hap.hap_moe_combine_bwd(d, j, Yj, di, pos, wd, g, dYd, dwd)
        hap.hap_moe_dispatch_bwd(d, j, dXj, di, pos, dxd)
        got = {n: host(t) for n, t in (("X", Xd), ("dY", dYd), ("out", outd), ("dx", dxd), ("dw", dwd))}
        for n in ("X", "dY", "out", "dx"):
            assert (got[n][..., h:] == SENTINEL).all(), n
        Xo = np.full((E, C, h), SENTINEL); dYo = Xo.copy()
        ort.dispatch_fwd(xh, idx, p, lo, hi, Xo)
        assert (got["X"][..., :h] == Xo[part]).all()
        w64 = w.astype(np.float64)
        terms = lambda a, b: ort.combine_fwd(np.abs(a), idx, p, np.abs(b), lo, hi)
        for n, ref, size in (("out", ort.combine_fwd(Yh, idx, p, w64, lo, hi), terms(Yh, w64)), ("dx", ort.dispatch_bwd(dXh, idx, p, lo, hi), terms(dXh, np.ones((T, k))))):
            err = np.abs(got[n][..., :h] - ref)
            assert (err <= HALF[dtype] * np.abs(ref) + 1.01 * (k + 1) * U * size).all(), (n, err.max())
        dwo = ort.combine_bwd(Yh, idx, p, w64, gh, lo, hi, dYo)
        err = np.abs(got["dY"][..., :h] - dYo[part])
        assert (err <= 1.01 * (HALF[dtype] + U) * np.abs(dYo[part]) * (dYo[part] != SENTINEL)).all()
        size = ort.combine_bwd(np.abs(Yh), idx, p, w64, np.abs(gh), lo, hi, np.zeros((E, C, h)))
        assert (np.abs(got["dw"] - dwo) <= 1.01 * (h / 64 + 9) * U * size).all()
    return p


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("T,k,E,C,h", [(1, 1, 1, 1, 1), (1, 2, 2, 1, 8), (5, 3, 7, 2, 64), (40, 2, 7, 9, 72), (33, 8, 64, 4, 520), (130, 1, 3, 50, 1024), (9, 64, 80, 7, 40), (17, 5, 3, 30, 1000)])
def test_tokens_round_trip(hap, dtype, full, T, k, E, C, h):
    """Devices with some, one and no experts; capacities that overflow; choices without an expert; NaN in rows without a token."""
    offs = [0, E // 2, E // 2, E]
    run_tokens(hap, dtype, T, k, E, C, h, offs, full, seed=T + h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_odd_rows_pitches_and_unaligned_views(hap, dtype):
    for h, pt, pe, shift in ((333, 0, 0, 0), (64, 1, 0, 0), (64, 0, 3, 0), (64, 8, 16, 0), (64, 8, 8, 1), (2, 0, 0, 0), (90, 6, 2, 2)):
        run_tokens(hap, dtype, 21, 2, 5, 6, h, [0, 3, 5], True, pt, pe, shift, seed=h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_rows_that_end_inside_a_chunk(hap, dtype):
    """Odd rows in pitches of whole chunks; the pitch's gaps hold NaN on the way in and must take no part in any sum."""
    torch = torch_mod()
    for h, ld, T, k, E, C in ((333, 336, 21, 2, 5, 6), (5, 8, 9, 3, 4, 5), (1021, 1024, 7, 1, 3, 9), (77, 96, 30, 4, 6, 12), (513, 520, 5, 2, 2, 5)):
        run_tokens(hap, dtype, T, k, E, C, h, [0, 2, E], True, ld - h, ld - h, seed=h)
        rng = np.random.default_rng(h)
        idx = np.argsort(rng.random((T, max(E, k))), axis=1)[:, :k]
        di, pos, _, _ = run_plan(hap, idx, E, C)
        p = pos.cpu().numpy()
        mk = lambda *shape: placed(rng.normal(size=shape), dtype, ld)
        (gh, g), (Yh, Y) = mk(T, h), mk(E, C, h)
        g[..., h:] = float("nan"); Y[..., h:] = float("nan")
        w = rng.normal(size=(T, k)).astype(np.float32)
        d = hap.MoeTokensDesc(T, k, E, C, h, [0, E], hap.BF16 if dtype == "bf16" else hap.F32, ld, ld)
        dw = torch.empty((T, k), device="cuda"); out = torch.zeros_like(g); dY = torch.zeros_like(Y)
        hap.hap_moe_combine_bwd(d, 0, Y, di, pos, torch.from_numpy(w).cuda(), g, dY, dw)
        hap.hap_moe_combine_fwd(d, 0, Y, di, pos, torch.from_numpy(w).cuda(), out)
        dwo = ort.combine_bwd(Yh, idx, p, w.astype(np.float64), gh, 0, E, np.zeros((E, C, h)))
        size = ort.combine_bwd(np.abs(Yh), idx, p, w.astype(np.float64), np.abs(gh), 0, E, np.zeros((E, C, h)))
        assert (np.abs(host(dw) - dwo) <= 1.01 * (h / 64 + 9) * U * size).all()
        assert (out[..., h:] == 0).all() and (dY[..., h:] == 0).all() and torch.isfinite(out).all()


def test_capacity_zero_and_empty_device(hap):
    """Nothing fits: the sums are zeros, nothing else is written; a device without experts owes zeros too."""
    torch = torch_mod()
    idx = torch.zeros((3, 2), dtype=torch.int32, device="cuda"); pos = torch.full_like(idx, -1)
    for C, offs, j in ((0, [0, 4], 0), (5, [0, 0, 4], 0)):
        d = hap.MoeTokensDesc(3, 2, 4, C, 16, offs, hap.BF16)
        out = torch.full((3, 16), 7.0, dtype=torch.bfloat16, device="cuda"); dx = out.clone(); w = torch.ones((3, 2), device="cuda"); dw = torch.full_like(w, 5.0)
        hap.hap_moe_combine_fwd(d, j, None, idx, pos, w, out)
        hap.hap_moe_dispatch_bwd(d, j, None, idx, pos, dx)
        hap.hap_moe_combine_bwd(d, j, None, idx, pos, w, out, None, dw)
        hap.hap_moe_dispatch_fwd(d, j, out, idx, pos, None)
        assert (out == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_positions_that_no_plan_gave_stay_inside(hap):
    """Positions and indices outside their ranges take no part: the buffer's neighbours stay as they were."""
    torch = torch_mod()
    E, C, h = 3, 4, 32
    idx = torch.tensor([[0, 5], [2, -3], [1, 2 ** 31 - 1], [-2 ** 31, 2]], dtype=torch.int32, device="cuda")
    pos = torch.tensor([[0, 0], [4, 1], [-5, 0], [2, 3]], dtype=torch.int32, device="cuda")
    d = hap.MoeTokensDesc(4, 2, E, C, h, [0, 3], hap.F32)
    guard = torch.full((E * C * h + 2048,), 7.0, device="cuda")
    X = guard[1024:-1024].view(E, C, h)
    x = torch.randn(4, h, device="cuda")
    hap.hap_moe_dispatch_fwd(d, 0, x, idx, pos, X)
    want = torch.full_like(X, 7.0); want[0, 0] = x[0]; want[2, 3] = x[3]
    assert torch.equal(X, want) and (guard[:1024] == 7).all() and (guard[-1024:] == 7).all()
    out = torch.empty_like(x)
    hap.hap_moe_combine_fwd(d, 0, X, idx, pos, torch.ones((4, 2), device="cuda"), out)
    assert torch.equal(out[0], x[0]) and torch.equal(out[3], x[3]) and (out[1:3] == 0).all()


def test_buffers_beyond_two_to_the_31_elements(hap):
    torch = torch_mod()
    E, C, h, T = 3, 190_000, 4096, 5                    # 2.3e9 elements
    X = torch.empty((E, C, h), dtype=torch.bfloat16, device="cuda")
    x = torch.randn(T, h, device="cuda").bfloat16()
    idx = torch.full((T, 1), 2, dtype=torch.int32, device="cuda")
    pos = torch.tensor([[0], [C - 1], [1], [C - 2], [7]], dtype=torch.int32, device="cuda")
    d = hap.MoeTokensDesc(T, 1, E, C, h, [0, E], hap.BF16)
    hap.hap_moe_dispatch_fwd(d, 0, x, idx, pos, X)
    assert torch.equal(X[2][pos[:, 0].long()], x)
    out = torch.empty_like(x); w = torch.ones((T, 1), device="cuda")
    hap.hap_moe_combine_fwd(d, 0, X, idx, pos, w, out)
    assert torch.equal(out, x)
    dw = torch.empty_like(w)
    dX = torch.empty_like(X)
    hap.hap_moe_combine_bwd(d, 0, X, idx, pos, 2 * w, x, dX, None)
    assert torch.equal(dX[2][pos[:, 0].long()], 2 * x)


@pytest.mark.parametrize("dtype,h", [("bf16", 4096), ("f32", 2048)])
def test_buffers_that_the_last_level_cache_does_not_hold(hap, dtype, h):
    """340 MB of buffer rows, moved there and back: rows and gradients are exact, rows without a token stay as they were, an overflowing expert included."""
    torch = torch_mod()
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    T, k, E, C = 5200, 8, 32, 1350
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    score = torch.rand((T, E), device="cuda", generator=gen); score[:, 5] += 0.6; score[:, 6] -= 0.6
    idx = score.argsort(dim=1, descending=True)[:, :k].int().contiguous()
    idx[7] = -1
    pos, rows = torch.empty_like(idx), torch.empty((E,), dtype=torch.int32, device="cuda")
    ws = torch.empty((max(hap.hap_moe_plan_workspace(T, k, E), 16),), dtype=torch.uint8, device="cuda")
    hap.hap_moe_plan(T, k, E, C, idx, pos, rows, None, ws)
    live = pos >= 0
    assert int(rows[5]) == C and int(rows.sum()) * h * (2 if dtype == "bf16" else 4) > 300 << 20
    d = hap.MoeTokensDesc(T, k, E, C, h, [0, E], hap.BF16 if dtype == "bf16" else hap.F32)
    x = torch.randint(-64, 65, (T, h), device="cuda", generator=gen).to(td)
    X = torch.full((E, C, h), SENTINEL, dtype=td, device="cuda")
    hap.hap_moe_dispatch_fwd(d, 0, x, idx, pos, X)
    e, p, t = idx[live].long(), pos[live].long(), live.nonzero()[:, 0]
    assert torch.equal(X[e, p], x[t])
    empty = torch.arange(C, device="cuda")[None, :] >= rows[:, None]
    assert (X[empty] == SENTINEL).all()
    w = torch.randint(-2, 3, (T, k), device="cuda", generator=gen).float()
    dX, dw, out = torch.full_like(X, SENTINEL), torch.empty_like(w), torch.empty_like(x)
    hap.hap_moe_combine_bwd(d, 0, X, idx, pos, w, x, dX, dw)
    assert torch.equal(dX[e, p], x[t] * w[live][:, None].to(td)) and (dX[empty] == SENTINEL).all()
    # whole numbers: sums below 2^24 are exact in fp32 whatever their order
    norm = (x.double() ** 2).sum(dim=1)
    assert torch.equal(dw.double(), torch.where(live, norm[:, None], torch.zeros_like(norm)[:, None]))
    hap.hap_moe_combine_fwd(d, 0, X, idx, pos, w, out)
    assert torch.equal(out, (x.double() * torch.where(live, w, torch.zeros_like(w)).double().sum(dim=1)[:, None]).to(td))
