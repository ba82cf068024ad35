"""The backward pass of the FFN on 4-bit weights: its definition on the CPU, refusals, and the GPU call against the oracle.

The definition passes the quantisations straight through, so all four gradients are those of a function in which Q(v) = v + a constant: the
oracle's are compared with difference quotients of that function.

The GPU's tolerances follow from its arithmetic, with u = 2^-8 (half a step of bfloat16) and a sum of n terms in fp32 off by at most
(n + 2) 2^-23 of the sum of their sizes.  dY, the saved G and U, the weights and Q(X) are exact inputs; Q(A) may be another value of its grid where A lies within
the forward pass's error of a border (`a_slack`, derived in test_mxfp4.py).
  dA    dots of H terms
  dG    dA U D, D = s + g s (1 - s) = silu'; s = 1 / (1 + e^-g) to r = (8 + 8 |g|) 2^-24 relative, so D to r (s + |g| s (1 - s) + |g| s^2) = r s (1 + |g|)
        and four roundings of terms that s (1 + |g|) bounds; the products four more; then rounded to bfloat16
  dU    dA g s likewise
  dX, dWg, dWu, dWd    sums of products with those, rounded once more.
"""
import numpy as np
import pytest
import torch

from oracle import dynmo_oracle as orc
from paper_2505_14864_amd import binding as B
from paper_2505_14864_amd.layer import RoutedFFNLayer

from test_mxfp4 import bf16, make_weights, segments

U8, V = 2.0 ** -8, 2.0 ** -24


def sums(n):
    return (n + 2) * 2.0 ** -23


def a_slack(x_p, seg, W, A, G, U):
    """How far the GPU's Q(A) may be from the oracle's, as test_mxfp4.py derives it."""
    xq = np.abs(orc.mxfp4_quantize(x_p)[0])
    steps = (-(-x_p.shape[1] // 128) + 2) * 2.0 ** -23
    dG, dU = np.zeros_like(G), np.zeros_like(U)
    for e in range(len(W[0])):
        rows = slice(int(seg[e]), int(seg[e + 1]))
        dG[rows], dU[rows] = steps * (xq[rows] @ np.abs(W[0][e]).T), steps * (xq[rows] @ np.abs(W[1][e]).T)
    dA = 1.1 * dG * np.abs(U) + np.abs(G * orc._sigmoid(G)) * dU + (8 + 8 * np.abs(G)) * V * np.abs(A)
    mid = orc.mxfp4_quantize(A)[0]
    high, _, s_high = orc.mxfp4_quantize(np.sign(A) * (np.abs(A) + dA))
    low, _, s_low = orc.mxfp4_quantize(np.sign(A) * np.maximum(np.abs(A) - dA, 0))
    unit = np.repeat(2.0 ** (s_high.astype(np.float64) - 127), 32, axis=-1)[:, :A.shape[1]]
    moved = np.repeat(s_high != s_low, 32, axis=-1)[:, :A.shape[1]]
    return np.maximum(np.abs(high - mid), np.abs(low - mid)) + np.where(moved, 2 * unit, 0)


def bounds(dy, x_p, seg, W, A, Gs, Us, slack, ref):
    """Tolerances of dX, dWg, dWu, dWd; Gs, Us as saved."""
    xq, aq = np.abs(orc.mxfp4_quantize(x_p)[0]), np.abs(orc.mxfp4_quantize(A)[0]) + slack
    s = orc._sigmoid(Gs)
    silu, D, r = np.abs(Gs * s), np.abs(s + Gs * s * (1 - s)), (8 + 8 * np.abs(Gs)) * V
    eD = (r + 4 * V) * s * (1 + np.abs(Gs))
    out = [np.zeros_like(t) for t in ref]
    H, F = x_p.shape[1], A.shape[1]
    for e in range(len(W[0])):
        rows = slice(int(seg[e]), int(seg[e + 1]))
        n = rows.stop - rows.start
        ady, dA = np.abs(dy[rows]), np.abs(dy[rows] @ W[2][e])
        eA = sums(H) * (ady @ np.abs(W[2][e]))
        u, dG, dU = np.abs(Us[rows]), dA * np.abs(Us[rows]) * D[rows], dA * silu[rows]
        eG = eA * u * (D[rows] + eD[rows]) + dA * u * eD[rows] + 4 * V * dG
        eU = (eA + dA * 3 * V) * silu[rows] * (1 + r[rows]) + dA * silu[rows] * r[rows]
        eG, eU = eG * (1 + U8) + U8 * dG, eU * (1 + U8) + U8 * dU
        out[0][rows] = eG @ np.abs(W[0][e]) + eU @ np.abs(W[1][e])
        out[0][rows] += sums(2 * F) * ((dG + eG) @ np.abs(W[0][e]) + (dU + eU) @ np.abs(W[1][e]))
        out[1][e] = (eG + sums(n) * (dG + eG)).T @ xq[rows]
        out[2][e] = (eU + sums(n) * (dU + eU)).T @ xq[rows]
        out[3][e] = ady.T @ (slack[rows] + sums(n) * aq[rows])
    return [t * (1 + U8) + U8 * np.abs(r) + 1e-30 for t, r in zip(out, ref)]


# ---- the definition ---------------------------------------------------------------------------------------------------------

def test_oracle_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((7, 40))
    W = [0.2 * rng.standard_normal(s) for s in ((3, 24, 40), (3, 24, 40), (3, 40, 24))]
    seg, dy = np.array([0, 4, 4, 7]), rng.standard_normal((7, 40))
    _, G, U, A = orc.grouped_ffn_mxfp4(x, seg, *W)
    cx, ca = orc.mxfp4_quantize(x)[0] - x, orc.mxfp4_quantize(A)[0] - A

    def loss(x, Wg, Wu, Wd):
        total = 0.0
        for e in range(3):
            rows = slice(seg[e], seg[e + 1])
            xq = x[rows] + cx[rows]
            g, u = xq @ Wg[e].T, xq @ Wu[e].T
            total += float((dy[rows] * ((g / (1 + np.exp(-g)) * u + ca[rows]) @ Wd[e].T)).sum())
        return total

    args = [x] + W
    grads = orc.grouped_ffn_mxfp4_bwd(dy, x, A, G, U, seg, *W)
    for i in range(4):
        for _ in range(40):
            at = tuple(rng.integers(0, n) for n in args[i].shape)
            step = np.zeros(args[i].shape)
            step[at] = 1e-5
            up, down = ([a + s * step if j == i else a for j, a in enumerate(args)] for s in (1, -1))
            assert abs((loss(*up) - loss(*down)) / 2e-5 - grads[i][at]) < 1e-7, (i, at)
    assert all((t[1] == 0).all() for t in grads[1:])  # the expert without rows


def test_the_tolerances_tell_the_gradients_of_unquantised_rows_apart():
    rng = np.random.default_rng(2)
    x = bf16(rng.standard_normal((64, 128))).float().numpy().astype(np.float64)
    W = [orc.mxfp4_quantize(rng.standard_normal(s) / np.sqrt(s[-1]))[0] for s in ((2, 160, 128), (2, 160, 128), (2, 128, 160))]
    seg, dy = np.array([0, 40, 64]), bf16(rng.standard_normal((64, 128))).float().numpy().astype(np.float64)
    _, G, U, A = orc.grouped_ffn_mxfp4(x, seg, *W)
    ref = orc.grouped_ffn_mxfp4_bwd(dy, x, A, G, U, seg, *W)
    tol = bounds(dy, x, seg, W, A, G, U, a_slack(x, seg, W, A, G, U), ref)
    plain = orc.grouped_ffn_bwd(dy, x, G, U, seg, *W)
    np.testing.assert_allclose(plain[0], ref[0], rtol=1e-9, atol=1e-12)
    for p, r, t in zip(plain[1:], ref[1:], tol[1:]):
        assert (np.abs(p - r) > t).mean() > 0.5


# ---- refusals ---------------------------------------------------------------------------------------------------------------

def test_refusals_without_a_gpu():
    ref, big = B.C.byref, 1 << 40
    d = B.make_desc(8, 16, 16, 4, 2, "bf16")
    names = ("dy_p", "G", "U", "seg", "Wg", "Wu", "Wd", "dx_p", "dWg", "dWu", "dWd", "saved", "ws")

    def call(desc=d, saved_bytes=big, bytes=big, **p):
        p = {n: p.get(n, 16) for n in names}
        return B.lib().dynmo_grouped_ffn_mxfp4_bwd(ref(desc), p["dy_p"], p["saved"], saved_bytes, p["G"], p["U"], p["seg"], p["Wg"], p["Wu"], p["Wd"],
                                                   p["dx_p"], p["dWg"], p["dWu"], p["dWd"], p["ws"], bytes, None)

    for name in names:
        assert call(**{name: None}) == -1, name
    for name in names[:3] + names[4:-2]:
        assert call(**{name: 24}) == -1, name
    assert call(saved_bytes=B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d) - 1) == -3
    assert call(bytes=B.dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(d) - 1) == -3
    assert call(desc=B.make_desc(8, 16, 16, 4, 2, "f32")) == -2 and call(desc=B.make_desc(8, (1 << 22) + 8, 16, 4, 2, "bf16")) == -2
    assert call(desc=B.make_desc(1 << 27, 8, 8, 4, 2, "bf16")) == -2 and call(desc=B.make_desc(8, 16, 16, 65, 2, "bf16")) == -2
    assert call(desc=B.make_desc(8, 16, 16, 4, 5, "bf16")) == -1
    assert B.dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(B.make_desc(8, 16, 16, 4, 2, "f32")) == 0
    assert B.dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(d) >= B.dynmo_grouped_ffn_bwd_workspace_bytes(d) + 16 * 16 * 2


@pytest.mark.parametrize("T,H,F,E", [(1 << 20, 8, 1 << 22, 4),   # gate/up
                                     (1 << 20, 1 << 22, 8, 4),   # the down product alone
                                     (1 << 14, 16, 1 << 22, 64), (1 << 14, 1 << 22, 16, 64)])
def test_too_many_tiles_are_refused_before_anything_is_launched(T, H, F, E):
    """Without a GPU a launch gives another error than the refusal."""
    d, room = B.make_desc(T, H, F, E, 1 if T > 1 << 14 else 16, "bf16"), 1 << 60
    fwd, bwd = B.lib().dynmo_grouped_ffn_mxfp4, B.lib().dynmo_grouped_ffn_mxfp4_bwd
    assert fwd(B.C.byref(d), 16, None, 16, 16, 16, 16, 16, None, None, 16, room, None) == -2
    assert bwd(B.C.byref(d), 16, 16, room, *[16] * 10, 16, room, None) == -2


# ---- the GPU ----------------------------------------------------------------------------------------------------------------

def at_offset(n, at):
    """n bytes that start `at` bytes into a buffer with 256 bytes behind them, and the whole buffer."""
    whole = torch.full((n + at + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    return whole[at:at + n], whole


def to_f64(t):
    return t.float().cpu().numpy().astype(np.float64)


CASES = [(1, 8, 8, 1, 1, [1]), (17, 136, 72, 2, 2, [20, 0]), (5, 520, 520, 3, 3, [0, 15, 0]), (40, 256, 640, 4, 2, [33, 0, 30, 17]),
         (150, 264, 136, 3, 2, [128, 129, 43]), (300, 392, 304, 5, 1, [0, 300, 0, 0, 0]), (70, 512, 1032, 64, 8, [9] * 62 + [0, 2]),
         (4, 64, 64, 3, 2, [0, 0, 0]), (16, 264, 136, 4, 4, [40, 0, 3, 20]),
         (256, 4096, 3584, 1, 1, [200])]  # the weight gradients' largest tiles


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,F,E,k,counts", CASES)
@pytest.mark.parametrize("gather", [False, True])
def test_ffn_bwd(T, H, F, E, k, counts, gather):
    rng = np.random.default_rng(T * 31 + H + F * 7 + E)
    R = int(sum(counts))
    packed, W = make_weights(E, H, F, rng)
    x = bf16(rng.standard_normal((T if gather else T * k, H)))
    dy = bf16(rng.standard_normal((T * k, H)))
    slots, seg = segments(counts, T, k, rng)
    src = torch.from_numpy(np.concatenate([slots, np.full(T * k - R, -1, np.int32)])).cuda() if gather else None
    d, seg_d = B.make_desc(T, H, F, E, k, "bf16"), torch.from_numpy(seg).cuda()
    act = dict(dtype=torch.bfloat16, device="cuda")
    y, G, U, dx = (torch.full((T * k, n), 7.0, **act) for n in (H, F, F, H))
    dW = [torch.full(s, 7.0, **act) for s in ((E, F, H), (E, F, H), (E, H, F))]
    saved, saved_whole = at_offset(B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d), 17)
    ws, ws_whole = at_offset(B.dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(d), 255)
    B.dynmo_grouped_ffn_mxfp4(d, x.cuda(), src, seg_d, *packed, y, G, U, saved)
    kept = saved_whole.clone()
    B.dynmo_grouped_ffn_mxfp4_bwd(d, dy.cuda(), saved, G, U, seg_d, *[torch.from_numpy(w).bfloat16().cuda() for w in W], dx, *dW, ws)
    assert torch.equal(kept, saved_whole)
    assert (ws_whole[:255] == 0x5A).all() and (ws_whole[-256:] == 0x5A).all()
    x_p = x.double().numpy()[slots // k] if gather else x.double().numpy()[:R]
    _, Ge, Ue, A = orc.grouped_ffn_mxfp4(x_p, seg, *W)
    Gs, Us, dyr = to_f64(G)[:R], to_f64(U)[:R], dy.double().numpy()[:R]
    ref = orc.grouped_ffn_mxfp4_bwd(dyr, x_p, A, Gs, Us, seg, *W)
    tol = bounds(dyr, x_p, seg, W, A, Gs, Us, a_slack(x_p, seg, W, A, Ge, Ue), ref)
    for name, got, r, t in zip(("dX", "dWg", "dWu", "dWd"), [dx[:R]] + dW, ref, tol):
        over = np.abs(to_f64(got) - r) - t
        assert not (over > 0).any(), (name, over.max(), (over > 0).sum())
    assert (to_f64(dx)[R:] == 7.0).all()  # rows behind the last segment are left as they were


@pytest.mark.gpu
def test_layer_gradients_of_the_weights():
    """All gradients as a layer runs them: routing with slots left out, the forward pass on packed weights, the backward pass."""
    T, H, F, E, k = 90, 128, 160, 8, 3
    rng = np.random.default_rng(12)
    packed, W = make_weights(E, H, F, rng)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    logits[:, 3], logits[5] = -np.inf, -np.inf  # an expert without rows, a token without experts
    x, dout = bf16(rng.standard_normal((T, H))), bf16(rng.standard_normal((T, H)))
    layer = RoutedFFNLayer(T, H, F, E, k, "bf16")
    layer.route_scored(torch.from_numpy(logits).cuda(), B.make_rule("sigmoid"))
    layer.forward_mxfp4(x.cuda(), *packed, train=True)
    dx = layer.backward(dout.cuda(), *[torch.from_numpy(w).bfloat16().cuda() for w in W])
    x_p, seg, _, dst = orc.permute(x.float().numpy(), layer.expert_idx.cpu().numpy(), E)[:4]
    R = int(seg[-1])
    assert 0 < R < T * k
    x_p = np.asarray(x_p[:R], np.float64)
    _, Ge, Ue, A = orc.grouped_ffn_mxfp4(x_p, seg, *W)
    Gs, Us, dyr = to_f64(layer.G)[:R], to_f64(layer.U)[:R], to_f64(layer.dy_p)[:R]
    ref = orc.grouped_ffn_mxfp4_bwd(dyr, x_p, A, Gs, Us, seg, *W)
    tol = bounds(dyr, x_p, seg, W, A, Gs, Us, a_slack(x_p, seg, W, A, Ge, Ue), ref)
    for name, got, r, t in zip(("dX", "dWg", "dWu", "dWd"), (layer.dx_p[:R], layer.dWg, layer.dWu, layer.dWd), ref, tol):
        over = np.abs(to_f64(got) - r) - t
        assert not (over > 0).any(), (name, over.max())
    assert (layer.dWd[3] == 0).all() and (dx[5] == 0).all()


@pytest.mark.gpu
def test_layer_backward_is_that_of_the_last_forward():
    T, H, F, E, k = 50, 128, 96, 4, 1
    rng = np.random.default_rng(3)
    packed, W = make_weights(E, H, F, rng)
    Wd = [torch.from_numpy(w).bfloat16().cuda() for w in W]
    x, dout = (bf16(rng.standard_normal((T, H))).cuda() for _ in range(2))
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    layer, other = (RoutedFFNLayer(T, H, F, E, k, "bf16") for _ in range(2))
    for l in (layer, other):
        l.route_topk(logits)
    layer.forward_mxfp4(x, *packed)
    for call in (layer.backward, layer.backward_folded):
        with pytest.raises(ValueError):  # nothing was kept
            call(dout, *Wd)
    layer.forward_mxfp4(x, *packed, train=True)
    with pytest.raises(ValueError):
        layer.backward_folded(dout, *Wd)
    layer.backward(dout, *Wd)
    of_quantised = layer.dWd.clone()
    for forward in ("forward", "forward_folded"):
        for l in (layer, other):
            getattr(l, forward)(x, *Wd)
            l.backward(dout, *Wd)
        for name in ("dx", "dWg", "dWu", "dWd"):
            assert torch.equal(getattr(layer, name), getattr(other, name)), name
        assert not torch.equal(layer.dWd, of_quantised)


@pytest.mark.gpu
def test_captured_step():
    """A training step on packed weights as a graph, replayed on other inputs, between eager ones on the same buffers."""
    T, H, F, E, k = 96, 256, 136, 4, 2
    rng = np.random.default_rng(6)
    packed, W = make_weights(E, H, F, rng)
    Wd = [torch.from_numpy(w).bfloat16().cuda() for w in W]
    layer = RoutedFFNLayer(T, H, F, E, k, "bf16")
    x, dout = (torch.zeros((T, H), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logits, rule = torch.zeros((T, E), dtype=torch.float32, device="cuda"), B.make_rule("softmax")

    def step():
        layer.route_scored(logits, rule)
        layer.forward_mxfp4(x, *packed, train=True)
        layer.backward(dout, *Wd)
        layer.route_bwd(logits)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (layer.out, layer.dx, layer.dWg, layer.dWu, layer.dWd, layer.droute)]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, dout, logits):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        replayed = results()
        step()
        for a, b in zip(replayed, results()):
            assert torch.equal(a, b)
