"""GPU tests of the routing, movement and expert operators run together, as a Mixture-of-Experts layer runs them: against the CPU oracle, over several virtual devices
whose partial results are added up, on other streams, and as HIP graphs that are replayed.

Tolerances as for the other layers: max|err| / max|ref| per tensor <= 2e-2 (bf16 in, fp32 accumulate) or 1e-5 (fp32).  The choice of experts follows the logits as the device rounded
them; they are compared on their own and handed to the oracle.
"""
import numpy as np
import pytest

from hapgen import TensorId as T_
from oracle import moe as omoe, routing as ort

pytestmark = pytest.mark.gpu

from gpu_util import gen, host, check, torch_mod  # noqa: E402


@pytest.fixture(scope="module")
def hap():
    import paper_2401_05965_amd as h
    return h


def make(dtype, T=300, h=96, F=160, E=7, seed=4):
    g = lambda tid, shape, sigma: gen(seed, tid, shape, sigma, dtype)
    t = dict(x=g(T_.X, (T, h), 1.0), dy=g(T_.DY, (T, h), 1.0), Wr=g(T_.WQ, (h, E), 0.1), W1=g(T_.W, (E, h, F), 0.1), b1=g(T_.BIAS, (E, F), 0.1), W2=g(T_.W2, (E, F, h), 0.1), b2=g(T_.BETA, (E, h), 0.1))
    return {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}


def layer(hap, d, offs, j, C, k, dtype, **route):
    from paper_2401_05965_amd.programs import MoeLayerShard
    torch = torch_mod()
    T, h = d["x"].shape
    E, _, F = d["W1"].shape
    return MoeLayerShard(T, h, F, E, C, k, offs, j, d["Wr"], d["W1"], d["b1"], d["W2"], d["b2"], dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, **route)


ROUTES = [dict(), dict(renormalise=False, scale=2.0), dict(score=1, renormalise=True, scale=1.5), dict(score=1, renormalise=False)]


def oracle_layer(v, logits, k, C, route, balance):
    sig, ren, sc = bool(route.get("score", 0)), route.get("renormalise", True), route.get("scale", 1.0)
    E = v["W1"].shape[0]
    idx, w = ort.route_fwd(logits, k, sig, balance, renormalise=ren, scale=sc)
    pos, rows, _ = ort.plan(idx, E, C)
    X = np.zeros((E, C, v["x"].shape[1]))
    ort.dispatch_fwd(v["x"], idx, pos, 0, E, X)
    H, pre = omoe.moe_linear_fwd(X, v["W1"], v["b1"], rows, True)
    Out, _ = omoe.moe_linear_fwd(H, v["W2"], v["b2"], rows, False)
    y = ort.combine_fwd(Out, idx, pos, w, 0, E)
    return dict(idx=idx, w=w, pos=pos, rows=rows, X=X, H=H, pre=pre, Out=Out, y=y)


def oracle_backward(v, logits, o, route):
    sig, ren, sc = bool(route.get("score", 0)), route.get("renormalise", True), route.get("scale", 1.0)
    E = v["W1"].shape[0]
    dOut = np.zeros_like(o["Out"])
    dw = ort.combine_bwd(o["Out"], o["idx"], o["pos"], o["w"], v["dy"], 0, E, dOut)
    dH, dW2, db2 = omoe.moe_linear_bwd(o["H"], v["W2"], None, dOut, o["rows"], False)
    dX, dW1, db1 = omoe.moe_linear_bwd(o["X"], v["W1"], o["pre"], dH, o["rows"], True)
    dl, _ = ort.route_bwd(logits, o["idx"], dw, sig, ren, sc)
    return dict(dx=ort.dispatch_bwd(dX, o["idx"], o["pos"], 0, E) + dl @ v["Wr"].T, dWr=v["x"].T @ dl, dW1=dW1, dW2=dW2, db1=db1, db2=db2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", range(len(ROUTES)))
def test_layer_over_uneven_devices(hap, dtype, which):
    """Seven experts on devices that hold 3, 0 and 4 of them; buffers that overflow; a balance bias with the sigmoid; partial results added up."""
    torch = torch_mod()
    route, k, C = ROUTES[which], 2, 80
    v, d = make(dtype)
    bal = (np.linspace(-0.2, 0.2, 7).astype(np.float32)) if route.get("score") else None
    bd = torch.from_numpy(bal).cuda() if bal is not None else None
    offs = [0, 3, 3, 7]
    parts = []
    for j in range(3):
        m = layer(hap, d, offs, j, C, k, dtype, balance=bd, **route)
        m.forward(d["x"]); m.backward(d["x"], d["dy"])
        parts.append(m)
    logits = host(parts[0].logits)[:, :7]
    check("logits", logits, v["x"] @ v["Wr"], dtype)
    o = oracle_layer(v, logits, k, C, route, bal.astype(np.float64) if bal is not None else None)
    assert (o["pos"] < 0).any() and (o["rows"] == C).any()                         # something overflows
    for m in parts:
        assert (m.indices.cpu().numpy() == o["idx"]).all() and (m.position.cpu().numpy() == o["pos"]).all() and (m.rows.cpu().numpy() == o["rows"]).all()
    check("y", sum(host(m.y) for m in parts), o["y"], dtype)
    b = oracle_backward(v, logits, o, route)
    check("dx", sum(host(m.dx) for m in parts), b["dx"], dtype)
    check("dWr", sum(host(m.dWr) for m in parts), b["dWr"], dtype)
    for n in ("dW1", "dW2", "db1", "db2"):
        check(n, np.concatenate([host(getattr(m.experts, n))[:m.experts.n] for m in parts]), b[n], dtype)
    # the norm over all devices' gradients (each listed once) and clipping by it
    total = torch.zeros((1,), dtype=torch.float64, device="cuda")
    lists = []
    for m in parts:
        shapes, grads = m.gradients()
        desc = hap.GradDesc(shapes, max_norm=0.5)
        one = torch.empty_like(total); ws = torch.empty((hap.hap_grad_sumsq_workspace(desc),), dtype=torch.uint8, device="cuda")
        hap.hap_grad_sumsq(desc, grads, one, ws)
        total += one
        lists.append((desc, grads))
    want = sum(float((g.double() ** 2).sum()) for _, gs in lists for g in gs)
    assert float(total) == pytest.approx(want, rel=1e-12)
    for desc, grads in lists:
        hap.hap_grad_clip(desc, grads, grads, total)
    after = sum(float((g.double() ** 2).sum()) for _, gs in lists for g in gs) ** 0.5
    assert after == pytest.approx(0.5, rel=2.0 ** -8)


def test_layer_gradient_against_differences(hap):
    """fp32: <dx, v> of the device against central differences of the oracle's forward along v, the choice held fixed.  The difference quotient is right to about step^2
    of the loss's third derivative and 1e-16 / step; the device's own error is the fp32 bar."""
    v, d = make("f32", T=60, h=32, F=48, E=5, seed=6)
    route, k, C = dict(renormalise=False, scale=2.0), 2, 40
    m = layer(hap, d, [0, 5], 0, C, k, "f32", **route)
    m.forward(d["x"]); m.backward(d["x"], d["dy"])
    idx = m.indices.cpu().numpy()

    def loss(x):
        logits = x @ v["Wr"]
        pos, rows, _ = ort.plan(idx, 5, C)
        w = np.stack([ort.weigh(logits[t], idx[t], False, False, 2.0) for t in range(60)])
        X = np.zeros((5, C, 32)); ort.dispatch_fwd(x, idx, pos, 0, 5, X)
        H, _ = omoe.moe_linear_fwd(X, v["W1"], v["b1"], rows, True)
        Out, _ = omoe.moe_linear_fwd(H, v["W2"], v["b2"], rows, False)
        return float((ort.combine_fwd(Out, idx, pos, w, 0, 5) * v["dy"]).sum())

    rng = np.random.default_rng(7)
    dx, step = host(m.dx), 1e-4
    for _ in range(4):
        u = rng.normal(size=v["x"].shape)
        num = (loss(v["x"] + step * u) - loss(v["x"] - step * u)) / (2 * step)
        assert abs((dx * u).sum() - num) <= 1e-5 * np.abs(dx).max() * np.abs(u).sum()


def test_layer_on_another_stream_and_two_at_once(hap):
    """Two layers of their own buffers and workspaces on two streams give the bits of one after the other."""
    torch = torch_mod()
    made = [make("bf16", T=500, h=256, F=128, E=8, seed=s)[1] for s in (1, 2)]
    ms = [layer(hap, d, [0, 8], 0, 160, 2, "bf16") for d in made]
    want = []
    for m, d in zip(ms, made):
        m.forward(d["x"]); m.backward(d["x"], d["dy"])
        torch.cuda.synchronize()
        want.append([t.clone() for t in (m.y, m.dx, m.dWr, m.weights, m.position)])
        for t in (m.y, m.dx, m.dWr, m.weights, m.position):
            t.fill_(7)
    streams = [torch.cuda.Stream() for _ in ms]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for m, d, s in zip(ms, made, streams):
            with torch.cuda.stream(s):
                m.forward(d["x"]); m.backward(d["x"], d["dy"])
    torch.cuda.synchronize()
    for m, w in zip(ms, want):
        for a, b in zip((m.y, m.dx, m.dWr, m.weights, m.position), w):
            assert torch.equal(a, b)


def test_training_step_as_a_graph(hap):
    """ids -> embedding -> layer -> gradients of layer and table -> norm -> clipping, captured once and replayed on new inputs, with eager work between the replays; every
    replay against the eager calls on the same inputs, bit for bit."""
    torch = torch_mod()
    T, h, F, E, V = 260, 128, 96, 6, 900
    _, d = make("bf16", T=T, h=h, F=F, E=E, seed=9)
    table = torch.randn(V, h, device="cuda").bfloat16()
    ids, x = torch.zeros((T,), dtype=torch.int64, device="cuda"), torch.zeros((T, h), dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros_like(x)
    emb = hap.EmbeddingDesc(T, V, h, hap.REPLICATED, None, hap.BF16, scale=2.0)
    ews = torch.empty((hap.hap_embedding_bwd_workspace(emb, 0),), dtype=torch.uint8, device="cuda")
    dtable = torch.zeros((V, h), device="cuda")
    m = layer(hap, d, [0, E], 0, 70, 2, "bf16", score=1, balance=torch.linspace(-0.1, 0.1, E, device="cuda"))
    shapes, grads = m.gradients()
    desc = hap.GradDesc(shapes + [(V, h, h, hap.F32)], max_norm=1.0)
    grads = grads + [dtable]
    gws = torch.empty((hap.hap_grad_sumsq_workspace(desc),), dtype=torch.uint8, device="cuda")
    total, norm = torch.zeros((1,), dtype=torch.float64, device="cuda"), torch.zeros((1,), device="cuda")

    def step():
        hap.hap_embedding_fwd(emb, 0, ids, table, x)
        m.forward(x); m.backward(x, dy)
        hap.hap_embedding_bwd(emb, 0, ids, m.dx, dtable, hap.F32, ws=ews)
        hap.hap_grad_sumsq(desc, grads, total, gws)
        hap.hap_grad_clip(desc, grads, grads, total, norm)

    outs = [x, m.y, m.dx, m.indices, m.position, m.weights, m.rows, m.counts, total, norm] + grads
    inputs = []
    for s in range(4):
        g = torch.Generator(device="cuda"); g.manual_seed(s)
        i = torch.randint(-3, V, (T,), device="cuda", generator=g)
        i[:50] = 11
        inputs.append((i, torch.randn(T, h, device="cuda", generator=g).bfloat16()))
    want = []
    for i, gy in inputs:
        ids.copy_(i); dy.copy_(gy)
        step()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for rep in range(2):
        for (i, gy), w in zip(inputs, want):
            for o in outs:
                o.fill_(3)
            ids.copy_(i); dy.copy_(gy)
            graph.replay()
            torch.cuda.synchronize()
            for n, (a, b) in enumerate(zip(outs, w)):
                assert torch.equal(a, b), (rep, n)
            (torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")).sum().item()


def test_workspaces_on_odd_words(hap):
    """Workspaces cut from a larger buffer one word behind a 256-byte boundary: the same bits as from its start."""
    torch = torch_mod()
    buf = torch.empty((1 << 23,), dtype=torch.uint8, device="cuda")
    idx = torch.randint(-1, 30, (20_000, 3), dtype=torch.int32, device="cuda")
    ids = torch.randint(-1, 500, (17_000,), device="cuda"); ids[:5000] = 7
    dY = torch.randn(17_000, 40, device="cuda")
    g = torch.randn(300, 500, device="cuda")
    E = hap.EmbeddingDesc(17_000, 500, 40, hap.REPLICATED, None, hap.F32)
    G = hap.GradDesc([(300, 500, 500, hap.F32)], 1.0)
    need = [hap.hap_moe_plan_workspace(20_000, 3, 30), hap.hap_embedding_bwd_workspace(E, 0), hap.hap_grad_sumsq_workspace(G)]
    assert min(need) > 0 and max(need) + 8 <= buf.numel()
    got = []
    for off in (0, 4):
        pos, rows = torch.empty_like(idx), torch.empty((30,), dtype=torch.int32, device="cuda")
        dW, total = torch.empty((500, 40), device="cuda"), torch.empty((1,), dtype=torch.float64, device="cuda")
        buf.fill_(255); hap.hap_moe_plan(20_000, 3, 30, 1500, idx, pos, rows, None, buf[off:off + need[0]])
        buf.fill_(255); hap.hap_embedding_bwd(E, 0, ids, dY, dW, hap.F32, ws=buf[off:off + need[1]])
        buf.fill_(255); hap.hap_grad_sumsq(G, [g], total, buf[2 * off:2 * off + need[2]])
        assert (buf[max(need) + 8:] == 255).all()
        got.append((pos, rows, dW, total))
    for a, b in zip(*got):
        assert torch.equal(a, b)
