"""Refusals of the routing, token movement, embedding and gradient-norm entry points: all on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest

EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED = 1, 2, 5, 7
P = 4096          # an address that is never used


@pytest.fixture(scope="module")
def hap():
    import paper_2401_05965_amd as h
    return h


def refused(hap, status, f, *args, **kw):
    with pytest.raises(hap.HapError) as e:
        f(*args, stream=0, **kw)
    assert e.value.status == status, str(e.value)


def test_route_refusals(hap):
    D = lambda **k: hap.RouteDesc(**{**dict(tokens=4, experts=8, top_k=2, io_dtype=hap.F32), **k})
    bad = [(EINVAL, dict(tokens=-1)), (EINVAL, dict(experts=0)), (EINVAL, dict(top_k=0)), (EINVAL, dict(score=2)), (EINVAL, dict(io_dtype=2)), (ESHAPE, dict(ld=7)), (ESHAPE, dict(top_k=9)),
           (EUNSUPPORTED, dict(experts=1025)), (EUNSUPPORTED, dict(experts=200, top_k=65)), (ESHAPE, dict(groups=3)), (ESHAPE, dict(groups=0)), (EINVAL, dict(groups=2, top_groups=3)),
           (EINVAL, dict(groups=2, top_groups=0)), (EINVAL, dict(groups=2, group_best=3)), (EINVAL, dict(group_best=0)), (ESHAPE, dict(groups=4, top_groups=1, top_k=3)),
           (EUNSUPPORTED, dict(experts=130, groups=65))]
    for status, k in bad:
        refused(hap, status, hap.hap_moe_route_fwd, D(**k), P, None, P, P)
        refused(hap, status, hap.hap_moe_route_bwd, D(**k), P, P, P, P)
    for i in range(3):
        a = [P, P, P]; a[i] = None
        refused(hap, EINVAL, hap.hap_moe_route_fwd, D(), a[0], None, a[1], a[2])
    for i in range(4):
        a = [P] * 4; a[i] = None
        refused(hap, EINVAL, hap.hap_moe_route_bwd, D(), *a)
    hap.hap_moe_route_fwd(D(tokens=0), None, None, None, None, stream=0)
    hap.hap_moe_route_bwd(D(tokens=0), None, None, None, None, stream=0)
    assert hap.lib.hap_moe_route_fwd(None, P, P, P, P, 0) == EINVAL


def test_plan_refusals(hap):
    f = hap.hap_moe_plan
    for status, a in ((EINVAL, (-1, 2, 8, 4)), (EINVAL, (4, 0, 8, 4)), (EINVAL, (4, 2, 0, 4)), (EINVAL, (4, 2, 8, -1)), (EUNSUPPORTED, (4, 2, 1025, 4)), (EUNSUPPORTED, (4, 65, 8, 4)),
                      (EUNSUPPORTED, (2 ** 30, 2, 8, 4)), (EUNSUPPORTED, (4, 2, 8, 2 ** 31))):
        refused(hap, status, f, *a, P, P, P)
    for i in range(3):
        p = [P] * 3; p[i] = None
        refused(hap, EINVAL, f, 4, 2, 8, 4, *p)
    need = hap.hap_moe_plan_workspace(100_000, 2, 8)
    assert need > 0 and hap.hap_moe_plan_workspace(4, 2, 8) == 0
    refused(hap, EWORKSPACE, f, 100_000, 2, 8, 4, P, P, P)
    assert hap.lib.hap_moe_plan(100_000, 2, 8, 4, P, P, P, P, P, need - 1, 0) == EWORKSPACE


def test_movement_refusals(hap):
    D = lambda offs=(0, 3, 8), **k: hap.MoeTokensDesc(**{**dict(tokens=4, top_k=2, experts=8, capacity=5, features=16, offsets=list(offs), io_dtype=hap.BF16), **k})
    calls = [lambda d, j=0, **n: hap.hap_moe_dispatch_fwd(d, j, n.get("t", P), n.get("i", P), n.get("p", P), n.get("e", P), stream=0),
             lambda d, j=0, **n: hap.hap_moe_dispatch_bwd(d, j, n.get("e", P), n.get("i", P), n.get("p", P), n.get("t", P), stream=0),
             lambda d, j=0, **n: hap.hap_moe_combine_fwd(d, j, n.get("e", P), n.get("i", P), n.get("p", P), n.get("w", P), n.get("t", P), stream=0),
             lambda d, j=0, **n: hap.hap_moe_combine_bwd(d, j, n.get("e", P), n.get("i", P), n.get("p", P), n.get("w", P), n.get("t", P), P, P, stream=0)]
    for which, call in enumerate(calls):
        for status, k in ((EINVAL, dict(tokens=-1)), (EINVAL, dict(features=0)), (EINVAL, dict(capacity=-1)), (EINVAL, dict(io_dtype=5)), (ESHAPE, dict(ldt=15)), (ESHAPE, dict(lde=15)),
                          (ESHAPE, dict(offs=(0, 3, 7))), (ESHAPE, dict(offs=(0, 9, 8))), (EUNSUPPORTED, dict(experts=1025, offs=(0, 1025))), (EUNSUPPORTED, dict(top_k=65)),
                          (EUNSUPPORTED, dict(capacity=2 ** 31)), (EUNSUPPORTED, dict(tokens=2 ** 30))):
            with pytest.raises(hap.HapError) as e:
                call(D(**k))
            assert e.value.status == status, (which, k, str(e.value))
        for j in (-1, 2):
            with pytest.raises(hap.HapError) as e:
                call(D(), j)
            assert e.value.status == EINVAL
        for missing in ("t", "i", "p", "e") + (("w",) if which > 1 else ()):
            with pytest.raises(hap.HapError) as e:
                call(D(), **{missing: None})
            assert e.value.status == EINVAL, (which, missing)
        call(D(tokens=0), t=None, i=None, p=None, e=None, w=None)      # no tokens: nothing to do


def test_embedding_refusals(hap):
    D = lambda offs=(0, 5, 16), **k: hap.EmbeddingDesc(**{**dict(tokens=9, vocab=16, hidden=16, mode=hap.SHARD_REDUCTION, offsets=list(offs), io_dtype=hap.BF16), **k})
    for status, k in ((EINVAL, dict(tokens=-1)), (EINVAL, dict(vocab=0)), (EINVAL, dict(hidden=0)), (EINVAL, dict(mode=4)), (EINVAL, dict(mode=-1)), (EINVAL, dict(io_dtype=3)), (EINVAL, dict(id_bytes=2)),
                      (ESHAPE, dict(ldw=15)), (ESHAPE, dict(ldy=15)), (ESHAPE, dict(offs=(0, 5, 15))), (EUNSUPPORTED, dict(tokens=2 ** 31)),
                      (EUNSUPPORTED, dict(hidden=2 ** 28)), (EUNSUPPORTED, dict(vocab=2 ** 30, mode=hap.REPLICATED))):
        refused(hap, status, hap.hap_embedding_fwd, D(**k), 0, P, P, P)
        refused(hap, status, hap.hap_embedding_bwd, D(**k), 0, P, P, P, hap.F32)
        assert hap.hap_embedding_bwd_workspace(D(**k), 0) == 0
    refused(hap, EINVAL, hap.hap_embedding_fwd, D(), 2, P, P, P)
    for i in range(3):
        a = [P] * 3; a[i] = None
        refused(hap, EINVAL, hap.hap_embedding_fwd, D(), 0, *a)
        refused(hap, EINVAL, hap.hap_embedding_bwd, D(), 0, *a, hap.F32)
    refused(hap, EINVAL, hap.hap_embedding_bwd, D(), 0, P, P, P, 7)
    refused(hap, EINVAL, hap.hap_embedding_bwd, D(io_dtype=hap.F32), 0, P, P, P, hap.BF16)
    refused(hap, EWORKSPACE, hap.hap_embedding_bwd, D(), 0, P, P, P, hap.F32)
    need = hap.hap_embedding_bwd_workspace(D(), 0)
    assert hap.lib.hap_embedding_bwd(C.byref(D().c), 0, P, P, P, hap.F32, 0, P, need - 1, 0) == EWORKSPACE
    empty = D(offs=(0, 0, 16))
    hap.hap_embedding_bwd(empty, 0, P, P, None, hap.F32, stream=0)            # a device without rows has no gradient
    hap.hap_embedding_fwd(D(tokens=0), 0, None, None, None, stream=0)


def test_grad_refusals(hap):
    D = lambda shapes=((2, 3, 4, 0), (1, 5, 5, 1)), max_norm=1.0: hap.GradDesc(shapes, max_norm)
    two = [P, P]
    for status, s in ((EINVAL, ((-1, 3, 4, 0), (1, 5, 5, 1))), (EINVAL, ((2, -3, 4, 0), (1, 5, 5, 1))), (EINVAL, ((2, 3, 4, 2), (1, 5, 5, 1))), (ESHAPE, ((2, 3, 2, 0), (1, 5, 5, 1))),
                      (EUNSUPPORTED, ((2 ** 31, 2 ** 31, 2 ** 31, 0), (1, 5, 5, 1))), (EUNSUPPORTED, ((2 ** 10, 2 ** 30, 2 ** 30, 0), (1, 1, 1, 0))), (EUNSUPPORTED, ((2, 2 ** 30, 2 ** 30 + 1, 0), (1, 1, 1, 0)))):
        refused(hap, status, hap.hap_grad_sumsq, D(s), two, P, None)
        refused(hap, status, hap.hap_grad_clip, D(s), two, two, P)
        assert hap.hap_grad_sumsq_workspace(D(s)) == 0
    for m in (0.0, -1.0, float("nan")):
        refused(hap, EINVAL, hap.hap_grad_clip, D(max_norm=m), two, two, P)
    refused(hap, EWORKSPACE, hap.hap_grad_sumsq, D(), two, P, None)
    refused(hap, EINVAL, hap.hap_grad_sumsq, D(), two, None, None)
    refused(hap, EINVAL, hap.hap_grad_sumsq, D(), [P, None], P, None)
    refused(hap, EINVAL, hap.hap_grad_clip, D(), [None, P], two, P)
    refused(hap, EINVAL, hap.hap_grad_clip, D(), two, [P, None], P)
    refused(hap, EINVAL, hap.hap_grad_clip, D(), two, two, None)
    refused(hap, ESHAPE, hap.hap_grad_clip, D(), two, [P + 64, P + 64], P, ldo=[2, 5])
    refused(hap, EINVAL, hap.hap_grad_clip, D(), two, two, P, ldo=[5, 5])     # in place with another pitch
    with pytest.raises(ValueError):
        hap.hap_grad_sumsq(D(), [P], P, None, stream=0)


def test_wrong_argument_types_are_type_errors(hap):
    with pytest.raises(TypeError):
        hap.hap_moe_plan(4.0, 2, 8, 4, P, P, P, stream=0)
    with pytest.raises(TypeError):
        hap.hap_embedding_fwd(hap.EmbeddingDesc(4, 4, 4, hap.REPLICATED, None, hap.F32), 0.5, P, P, P, stream=0)


def test_batches_beyond_a_grid_are_refused(hap):
    """A grid has fewer than 2^32 threads: with 256 threads for a workgroup, fewer than 2^24 workgroups."""
    most = 4 * 2 ** 24                                       # tokens, four of them a workgroup
    R = hap.RouteDesc(most, 1024, 1, hap.BF16)
    refused(hap, EUNSUPPORTED, hap.hap_moe_route_fwd, R, P, None, P, P)
    refused(hap, EUNSUPPORTED, hap.hap_moe_route_bwd, R, P, P, P, P)
    M = hap.MoeTokensDesc(most, 1, 8, 4, 16, [0, 8], hap.BF16)
    refused(hap, EUNSUPPORTED, hap.hap_moe_dispatch_fwd, M, 0, P, P, P, P)
    refused(hap, EUNSUPPORTED, hap.hap_moe_dispatch_bwd, M, 0, P, P, P, P)
    refused(hap, EUNSUPPORTED, hap.hap_moe_combine_fwd, M, 0, P, P, P, P, P)
    refused(hap, EUNSUPPORTED, hap.hap_moe_combine_bwd, M, 0, P, P, P, P, P, P, P)
    E = hap.EmbeddingDesc(most, 16, 8, hap.REPLICATED, None, hap.BF16)
    refused(hap, EUNSUPPORTED, hap.hap_embedding_fwd, E, 0, P, P, P)
    # the gradient: a workgroup for each chunk of 64 sorted tokens and slab of columns
    E = hap.EmbeddingDesc(2 ** 31 - 1, 16, 8, hap.REPLICATED, None, hap.BF16)
    need = hap.hap_embedding_bwd_workspace(E, 0)
    assert hap.lib.hap_embedding_bwd(C.byref(E.c), 0, P, P, P, hap.F32, 0, P, need, 0) == EUNSUPPORTED


@pytest.mark.parametrize("n", [2, 5, 300])
def test_clipping_one_output_twice_is_refused(hap, n):
    address = [P * (i + 1) for i in range(n)]
    address[-1] = address[0]
    d = hap.GradDesc(((2, 3, 3, hap.F32),) * n, 1.0)
    refused(hap, EINVAL, hap.hap_grad_clip, d, address, address, P)                          # a shared tensor that is listed twice
    refused(hap, EINVAL, hap.hap_grad_clip, d, [P * (i + 1000) for i in range(n)], address, P)


def test_workspaces_off_their_words_are_refused(hap):
    """Counts and keys are 32-bit words, partial sums of squares are doubles: a workspace cut from a larger buffer starts on a multiple of them."""
    E = hap.EmbeddingDesc(9, 16, 16, hap.REPLICATED, None, hap.BF16)
    G = hap.GradDesc(((2, 3, 3, hap.F32), (1, 5, 5, hap.F32)), 1.0)
    need = [hap.hap_moe_plan_workspace(100_000, 2, 8), hap.hap_embedding_bwd_workspace(E, 0), hap.hap_grad_sumsq_workspace(G)]
    two = (C.c_uint64 * 2)(P, P)
    calls = [lambda ws, n: hap.lib.hap_moe_plan(100_000, 2, 8, 4, P, P, P, P, ws, n, 0), lambda ws, n: hap.lib.hap_embedding_bwd(C.byref(E.c), 0, P, P, P, hap.F32, 0, ws, n, 0),
             lambda ws, n: hap.lib.hap_grad_sumsq(C.byref(G.c), two, P, ws, n, 0)]
    for call, n, word in zip(calls, need, (4, 4, 8)):
        assert n > 0
        for off in range(1, word):
            assert call(P + off, n) == EINVAL, (word, off)
        assert call(P + 1, n - 1) == EWORKSPACE
