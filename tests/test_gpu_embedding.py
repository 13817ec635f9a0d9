"""GPU parity of the embedding table and its gradient against the CPU oracle, for the four sharding rules.

u = 2^-24.  A looked-up value is one product: half a step of its type (and u before it, for bf16).  A gradient value is a sum over the n tokens of its id in some
fixed order, the scale and, accumulating, the old value: (n + 4) u of its terms' magnitudes, and half a step of its type.
"""
import numpy as np
import pytest

from oracle import embedding as oemb

pytestmark = pytest.mark.gpu

from gpu_util import host, torch_mod  # noqa: E402

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
SENTINEL = 768.0


@pytest.fixture(scope="module")
def hap():
    import paper_2401_05965_amd as h
    return h


def placed(values, dtype, ld, shift=0):
    torch = torch_mod()
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    R, n = values.shape
    buf = torch.full((R * ld + shift,), SENTINEL, dtype=td, device="cuda")
    view = buf[shift:].view(R, ld)
    view[:, :n] = torch.from_numpy(np.ascontiguousarray(values)).to(td).cuda()
    return view[:, :n].double().cpu().numpy(), view


def run_embedding(hap, mode, dtype, grad, T, V, h, offs, full, accumulate, id_bytes=8, ids=None, scale=2.0, pw=0, py=0, shift=0, seed=0):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    if ids is None:
        ids = np.minimum((V + 1) ** rng.random(T) - 1, V - 1).astype(np.int64)
        bad = rng.random(T) < 0.1
        ids[bad] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31] if id_bytes == 4 else [-100, V, 2 ** 40, -2 ** 63], bad.sum())
    type_ = {"bf16": hap.BF16, "f32": hap.F32}
    idd = torch.from_numpy(ids.astype(np.int32 if id_bytes == 4 else np.int64)).cuda()
    ldw, ldy = h + pw, h + py
    Wh, W = placed(rng.normal(size=(V, h)), dtype, ldw, shift)
    gh, g = placed(rng.normal(size=(T, h)), dtype, ldy, shift)
    old = rng.normal(size=(V, h))
    for j in range(len(offs) - 1 if mode != hap.REPLICATED else 1):
        lo, hi = (offs[j], offs[j + 1]) if mode != hap.REPLICATED else (0, 0)
        t = slice(lo, hi) if mode == hap.SHARD_BATCH else slice(0, T)
        v = slice(lo, hi) if mode == hap.SHARD_REDUCTION else slice(0, V)
        c = slice(lo, hi) if mode == hap.SHARD_FEATURE else slice(0, h)
        cut = lambda x, r, cc: x if full else x[r, cc.start:].contiguous() if mode == hap.SHARD_FEATURE else x[r]
        n_c = c.stop - c.start
        d = hap.EmbeddingDesc(T, V, h, mode, offs, type_[dtype], scale=scale, id_bytes=id_bytes, ldw=ldw if full or mode != hap.SHARD_FEATURE else ldw - c.start,
                              ldy=ldy if full or mode != hap.SHARD_FEATURE else ldy - c.start, operands_are_full=full)
        Y = cut(placed(np.full((T, h), SENTINEL), dtype, ldy, shift)[1], t, c)
        oldh, dW = placed(old, grad, ldw, shift)
        before = dW.clone()
        dW = cut(dW, v, c)
        i = idd if full else idd[t]
        hap.hap_embedding_fwd(d, j, i, cut(W, v, c), Y)
        ws = torch.empty((max(hap.hap_embedding_bwd_workspace(d, j), 16),), dtype=torch.uint8, device="cuda").fill_(255)
        hap.hap_embedding_bwd(d, j, i, cut(g, t, c), dW, type_[grad], accumulate, ws)
        # the unsharded oracle, cut to what the device owns
        mine = ids.copy()
        if mode == hap.SHARD_REDUCTION:
            mine = np.where((ids >= lo) & (ids < hi), ids, -1)
        ref = oemb.embedding_fwd(mine, Wh, scale)[t, c]
        gt = gh.copy()
        if mode == hap.SHARD_BATCH:
            out_of = np.ones(T, bool); out_of[t] = False
            gt[out_of] = 0
        dref, size = oemb.embedding_bwd(mine, gt, V, scale)
        n = np.bincount(mine[(mine >= 0) & (mine < V)], minlength=V)[:, None]
        Yh, dWh = host(Y), host(dW)
        if full:
            Yc, dWc = Yh[t, c], dWh[v, c]
            keep = np.ones(Yh.shape, bool); keep[t, c] = False
            assert (Yh[keep] == SENTINEL).all()
            keep = np.ones(dWh.shape, bool); keep[v, c] = False
            assert (dWh[keep] == host(before)[keep]).all()
        else:
            Yc, dWc = Yh[:, :n_c], dWh[:, :n_c]
            assert (Yh[:, n_c:] == SENTINEL).all() or mode == hap.SHARD_FEATURE
            if mode != hap.SHARD_FEATURE:
                assert (dWh[:, n_c:] == SENTINEL).all()
        assert (np.abs(Yc - ref) <= 1.01 * (HALF[dtype] + U) * np.abs(ref)).all()
        dref, size, n = dref[v, c], size[v, c], n[v]
        if accumulate:
            o = oldh[v, c]
            dref, size = dref + o, size + np.abs(o)
            assert (dWc[n[:, 0] == 0] == o[n[:, 0] == 0]).all()
        else:
            assert (dWc[n[:, 0] == 0] == 0).all()
        err = np.abs(dWc - dref)
        assert (err <= 1.01 * (HALF[grad] * np.abs(dref) + (n + 4) * U * size)).all(), err.max()


TYPES = [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")]


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("T,V,h", [(1, 1, 1), (1, 5, 8), (3, 1000, 64), (31, 7, 136), (32, 40, 64), (33, 40, 72), (64, 300, 520), (65, 511, 512), (500, 513, 40), (2100, 900, 33), (300, 2, 1024)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_sizes(hap, dtype, grad, T, V, h, accumulate):
    run_embedding(hap, hap.REPLICATED, dtype, grad, T, V, h, None, True, accumulate, seed=T + V)


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("mode", ["batch", "feature", "reduction"])
def test_embedding_sharding_rules(hap, dtype, grad, full, mode):
    """Three devices, one of them with nothing; ids of both widths; whole tensors and compact parts."""
    T, V, h = 150, 260, 144
    m, n = {"batch": (hap.SHARD_BATCH, T), "feature": (hap.SHARD_FEATURE, h), "reduction": (hap.SHARD_REDUCTION, V)}[mode]
    for a in (n // 3, 48):
        run_embedding(hap, m, dtype, grad, T, V, h, [0, a, a, n], full, False, id_bytes=4 if a == 48 else 8, seed=a)
    run_embedding(hap, m, dtype, grad, T, V, h, [0, 48, 48, n], full, True, seed=5)


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_columns_that_begin_and_end_inside_a_chunk(hap, dtype, grad, accumulate):
    """Uneven column ranges of whole tensors, and compact parts of odd width in pitches of whole chunks."""
    for h, pad, cuts in ((144, 0, (37, 38)), (144, 0, (50, 101)), (141, 3, (64, 65)), (520, 8, (3, 517)), (31, 1, (8, 13))):
        run_embedding(hap, hap.SHARD_FEATURE, dtype, grad, 120, 60, h, [0, *cuts, h], True, accumulate, pw=pad, py=pad, seed=h + cuts[0])
        run_embedding(hap, hap.REPLICATED, dtype, grad, 120, 60, h, None, True, accumulate, pw=pad, py=pad, seed=h)
    for h, pad in ((333, 3), (2731, 5), (5, 3), (1, 7)):
        run_embedding(hap, hap.REPLICATED, dtype, grad, 70, 40, h, None, True, accumulate, pw=pad, py=pad, seed=h)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_embedding_pitches_and_unaligned_views(hap, dtype, grad):
    for h, pw, py, shift in ((64, 8, 16, 0), (64, 1, 0, 0), (64, 0, 3, 0), (64, 8, 8, 1), (63, 1, 1, 0), (2, 0, 0, 3)):
        run_embedding(hap, hap.REPLICATED, dtype, grad, 90, 50, h, None, True, False, pw=pw, py=py, shift=shift, seed=h)


@pytest.mark.parametrize("T", [20, 33, 64, 97, 1500, 16384, 16385, 70001])
def test_embedding_gradient_of_one_id_and_of_runs(hap, T):
    """All tokens one id; two ids; an id that fills chunks exactly, with others at its borders; all padding; descending order; one workgroup's sort and many's."""
    V, h = 700, 16
    rng = np.random.default_rng(T)
    blocks = np.sort(np.repeat(np.arange(T // 32 + 1), 32)[:T] % V)
    for ids in (np.full(T, 3), rng.integers(0, 2, T) * (V - 1), blocks, np.full(T, -1), np.arange(T)[::-1] % V, np.where(np.arange(T) < T // 2, 5, 6)):
        run_embedding(hap, hap.REPLICATED, "f32", "f32", T, V, h, None, True, False, ids=ids.astype(np.int64), seed=1)


def test_embedding_gradient_over_large_tables_is_exact_for_whole_numbers(hap):
    """Three digits of sorting, more tokens than one workgroup sorts; whole-number gradients, so that any order gives the same bits."""
    torch = torch_mod()
    for T, V, h in ((5000, 300_001, 24), (50_000, 262_143, 16), (40_000, 262_144, 16), (16384, 1_000_003, 8)):
        gen = torch.Generator(device="cuda"); gen.manual_seed(V)
        ids = (torch.rand(T, device="cuda", generator=gen, dtype=torch.float64) ** 3 * V).long()
        ids[::17] = -1; ids[5] = V - 1; ids[6] = 0
        dY = torch.randint(-8, 9, (T, h), device="cuda", generator=gen).float()
        d = hap.EmbeddingDesc(T, V, h, hap.REPLICATED, None, hap.F32)
        dW = torch.full((V, h), 5.0, device="cuda")
        ws = torch.empty((hap.hap_embedding_bwd_workspace(d, 0),), dtype=torch.uint8, device="cuda")
        hap.hap_embedding_bwd(d, 0, ids, dY, dW, hap.F32, ws=ws)
        want = torch.zeros((V, h), dtype=torch.float64, device="cuda").index_add_(0, ids[ids >= 0], dY[ids >= 0].double())
        assert torch.equal(dW.double(), want)


def test_embedding_gradient_has_the_same_bits_in_every_run(hap):
    torch = torch_mod()
    T, V, h = 20_000, 900, 264
    ids = torch.randint(0, V, (T,), device="cuda"); ids[:9000] = 17
    dY = torch.randn(T, h, device="cuda").bfloat16()
    d = hap.EmbeddingDesc(T, V, h, hap.REPLICATED, None, hap.BF16)
    ws = torch.empty((hap.hap_embedding_bwd_workspace(d, 0),), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(4):
        dW = torch.empty((V, h), device="cuda")
        hap.hap_embedding_bwd(d, 0, ids, dY, dW, hap.F32, ws=ws)
        first = dW if first is None else first
        assert torch.equal(dW, first)


def test_embedding_of_no_tokens(hap):
    torch = torch_mod()
    d = hap.EmbeddingDesc(0, 9, 8, hap.REPLICATED, None, hap.F32)
    dW = torch.full((9, 8), 5.0, device="cuda")
    hap.hap_embedding_fwd(d, 0, None, dW, None)
    hap.hap_embedding_bwd(d, 0, None, None, dW, hap.F32, accumulate=True)
    assert (dW == 5).all()
    hap.hap_embedding_bwd(d, 0, None, None, dW, hap.F32)
    assert (dW == 0).all()
    dW = torch.full((300_000, 8), 5.0, device="cuda")
    hap.hap_embedding_bwd(hap.EmbeddingDesc(0, 300_000, 8, hap.REPLICATED, None, hap.F32), 0, None, None, dW, hap.F32)
    assert (dW == 0).all()


def test_tables_beyond_two_to_the_31_elements(hap):
    torch = torch_mod()
    V, h, T = 600_000, 4096, 6                         # 2.5e9 elements
    W = torch.empty((V, h), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, 524_288, V - 1, 3], device="cuda")
    W[ids] = torch.randn(T, h, device="cuda").bfloat16()
    d = hap.EmbeddingDesc(T, V, h, hap.REPLICATED, None, hap.BF16)
    Y = torch.empty((T, h), dtype=torch.bfloat16, device="cuda")
    hap.hap_embedding_fwd(d, 0, ids, W, Y)
    assert torch.equal(Y, W[ids])
    dW = W
    dW[ids[2] + 1] = 3.0; dW[V // 2] = 3.0
    ws = torch.empty((hap.hap_embedding_bwd_workspace(d, 0),), dtype=torch.uint8, device="cuda")
    hap.hap_embedding_bwd(d, 0, ids, Y, dW, hap.BF16, ws=ws)
    assert torch.equal(dW[V - 1], (Y[0].float() + Y[4].float()).bfloat16()) and torch.equal(dW[524_288], Y[3]) and torch.equal(dW[V - 2], Y[2])
    assert (dW[V // 2] == 0).all() and (dW[V - 5:V - 2] == 0).all() and int((dW != 0).any(dim=1).sum()) == 5


@pytest.mark.parametrize("dtype,h", [("bf16", 5120), ("f32", 2048)])
def test_lookups_that_the_caches_do_not_hold(hap, dtype, h):
    """90 MB of looked-up rows: the table's rows times a power of two exactly, zeros for padding; whole rows and columns that begin inside a chunk."""
    torch = torch_mod()
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    V = 3001
    T = 90_000_000 // (h * (2 if dtype == "bf16" else 4)) + 1
    gen = torch.Generator(device="cuda"); gen.manual_seed(h)
    W = torch.randn((V, h), device="cuda", generator=gen).to(td)
    ids = torch.randint(-50, V + 50, (T,), device="cuda", generator=gen)
    here = (ids >= 0) & (ids < V)
    want = torch.where(here[:, None], 2 * W[ids.clamp(0, V - 1)], torch.zeros((), dtype=td, device="cuda"))
    io = hap.BF16 if dtype == "bf16" else hap.F32
    Y = torch.full((T, h), SENTINEL, dtype=td, device="cuda")
    hap.hap_embedding_fwd(hap.EmbeddingDesc(T, V, h, hap.REPLICATED, None, io, scale=2.0), 0, ids, W, Y)
    assert torch.equal(Y, want)
    Y.fill_(SENTINEL)
    d = hap.EmbeddingDesc(T, V, h, hap.SHARD_FEATURE, [0, 8, h - 3, h], io, scale=2.0)
    for j in range(3):
        hap.hap_embedding_fwd(d, j, ids, W, Y)
    assert torch.equal(Y, want)
