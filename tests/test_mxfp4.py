"""Experts in 4 bits: pins of the oracle's quantisation and packed form, refusals, and the GPU calls against the oracle.

Quantisation is exact arithmetic: codes, scales and values have to be equal.  The FFN's tolerance follows from its arithmetic.  Products
of 4-bit values are exact in fp32; a product over K is ceil(K / 128) instructions, each of which was seen to add at most
2^-23 of the sum of the terms' sizes, so |dG| <= (ceil(K / 128) + 2) 2^-23 sum |x| |w|, U likewise; with silu' at most 1.1
and the logistic function to (8 + 8 |G|) 2^-24, |dA| follows.  Where A +- dA quantises to other values than A, Y may differ by that
difference times the weight (a block whose scale may change: by up to two units of the larger scale); to that come the last product's own sums and
the rounding to bf16, half a step: 2^-8.
"""
import numpy as np
import pytest
import torch

from oracle import dynmo_oracle as orc
from paper_2505_14864_amd import binding as B
from paper_2505_14864_amd.layer import RoutedFFNLayer

BF16 = 2.0 ** -8


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16()


# ---- the oracle's pins -----------------------------------------------------------------------------------------------------

def test_oracle_quantization_by_hand():
    x = np.zeros((1, 40))
    x[0, :12] = [6.0, -7.9, 0.25, 0.26, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -0.1]  # largest 7.9: scale 1
    x[0, 32:35] = [1.0, 0.0625, 0.07]                                                 # scale 1 / 4
    v, code, scale = orc.mxfp4_quantize(x)
    assert v[0, :12].tolist() == [6, -6, 0, 0.5, -1, 1, 2, 2, 4, 4, 6, 0]
    assert v[0, 32:35].tolist() == [1, 0, 0.125]
    assert code[0, 0, :12].tolist() == [7, 15, 0, 1, 10, 2, 4, 4, 6, 6, 7, 8]
    assert scale[0].tolist() == [127, 125] and code[0, 1, 8:].max() == 0
    v, code, scale = orc.mxfp4_quantize(np.array([[2.0 ** -126, 0], [0, 0], [np.inf, 1], [1, np.nan]]))
    assert scale[:, 0].tolist() == [0, 0, 255, 255] and np.isnan(v[2:]).all()
    assert v[0, 0] == 2.0 ** -126 and v[1, 0] == 0


def test_oracle_quantization_against_a_search():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((20, 96)) * np.exp(rng.standard_normal((20, 96)) * 2)
    v, _, scale = orc.mxfp4_quantize(x)
    for r in range(20):
        for b in range(3):
            blk, unit = x[r, 32 * b:32 * b + 32], 2.0 ** (int(scale[r, b]) - 127)
            assert 4 * unit <= np.abs(blk).max() < 8 * unit
            grid = np.concatenate([orc.MXFP4_VALUES, -orc.MXFP4_VALUES]) * unit
            best = np.abs(blk[:, None] - grid[None, :]).min(1)
            np.testing.assert_allclose(np.abs(v[r, 32 * b:32 * b + 32] - blk), best, rtol=1e-12)
    again, _, _ = orc.mxfp4_quantize(v)
    assert np.array_equal(again, v)  # quantising quantised values changes nothing


def test_oracle_packed_form_by_hand():
    codes = np.zeros((17, 17, 32), np.uint8)
    scales = np.zeros((17, 17), np.uint8)
    codes[16, 5, 6], codes[16, 5, 7] = 3, 9  # row 16: second row block; k = 166, 167: second tile, block 1
    scales[16, 16] = 77                      # k = 512: second quad, tile 0, block 0
    p = orc.mxfp4_pack(codes, scales)
    assert p.size == 2 * 5 * 1024 + 2 * 2 * 256
    assert p[(1 * 5 + 1) * 1024 + 1 * 256 + 0 * 16 + 3] == 3 + 9 * 16
    assert p[2 * 5 * 1024 + (1 * 2 + 1) * 256] == 77
    assert np.count_nonzero(p) == 2


def test_oracle_ffn_without_rounding_is_the_ffn():
    """Operands that lie on the grid pass the first products unchanged, and the quantised A is what the last one takes."""
    rng = np.random.default_rng(3)
    x = rng.choice([-3.0, -1.0, 0.5, 2.0, 6.0], size=(9, 64))
    W = [orc.mxfp4_quantize(0.1 * rng.standard_normal(s))[0] for s in ((3, 32, 64), (3, 32, 64), (3, 64, 32))]
    seg = np.array([0, 4, 4, 9])
    Y, G, U, A = orc.grouped_ffn_mxfp4(x, seg, *W)
    ref = orc.grouped_ffn_fwd(x, seg, *W)
    np.testing.assert_allclose(G, ref[1], rtol=1e-12)
    np.testing.assert_allclose(U, ref[2], rtol=1e-12)
    np.testing.assert_allclose(Y[5], orc.mxfp4_quantize(A)[0][5] @ W[2][2].T, rtol=1e-12)


# ---- refusals ----------------------------------------------------------------------------------------------------------------

def test_refusals_without_a_gpu():
    lib, ref = B.lib(), B.C.byref
    assert B.dynmo_mxfp4_bytes(16, 128) == 1024 + 256 and B.dynmo_mxfp4_bytes(17, 513) == 2 * 5 * 1024 + 2 * 2 * 256
    assert B.dynmo_mxfp4_bytes(0, 8) == 0 and B.dynmo_mxfp4_bytes(-1, 8) == 0 and B.dynmo_mxfp4_bytes(4, 0) == 0
    for call in (lib.dynmo_mxfp4_quantize, lib.dynmo_mxfp4_dequantize):
        assert call(1, 4, 8, 1, None, 16, None) == -1 and call(1, 4, 8, 1, 16, None, None) == -1
        assert call(1, 4, 8, 2, 16, 16, None) == -1 and call(-1, 4, 8, 1, 16, 16, None) == -1
        assert call(1, -4, 8, 1, 16, 16, None) == -1 and call(1, 4, 0, 1, 16, 16, None) == -1
        assert call(1, 4, 12, 1, 16, 16, None) == -2 and call(1, 4, 6, 0, 16, 16, None) == -2
        assert call(1, 4, 8, 1, 16, 24, None) == -1 and call(1, 4, 8, 1, 24, 16, None) == -1
        assert call(1 << 20, 1 << 20, 8, 1, 16, 16, None) == -2 and call(1, 1 << 28, 8, 1, 16, 16, None) == -2
        assert call(0, 4, 8, 1, None, None, None) == 0 and call(3, 0, 8, 1, None, None, None) == 0
    ffn, big = lib.dynmo_grouped_ffn_mxfp4, 1 << 40
    d = B.make_desc(8, 16, 16, 4, 2, "bf16")

    def call(desc=d, x=16, src=None, seg=16, Wg=16, Wu=16, Wd=16, y=16, G=None, U=None, ws=16, n=big):
        return ffn(ref(desc), x, src, seg, Wg, Wu, Wd, y, G, U, ws, n, None)

    for name in ("x", "seg", "Wg", "Wu", "Wd", "y", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("x", "Wg", "Wu", "Wd", "y"):
        assert call(**{name: 24}) == -1, name
    assert call(G=16) == -1 and call(U=16) == -1 and call(G=24, U=16) == -1
    assert call(n=B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d) - 1) == -3
    assert call(desc=B.make_desc(8, 16, 16, 4, 2, "f32")) == -2
    assert call(desc=B.make_desc(8, (1 << 22) + 8, 16, 4, 2, "bf16")) == -2
    assert call(desc=B.make_desc(1 << 27, 8, 8, 4, 2, "bf16")) == -2  # 2^24 row blocks
    assert call(desc=B.make_desc(8, 16, 16, 65, 2, "bf16")) == -2 and call(desc=B.make_desc(8, 12, 16, 4, 2, "bf16")) == -2
    assert call(desc=B.make_desc(8, 16, 16, 4, 5, "bf16")) == -1
    assert B.dynmo_grouped_ffn_mxfp4_workspace_bytes(B.make_desc(8, 16, 16, 4, 2, "f32")) == 0
    assert call(desc=B.make_desc(0, 16, 16, 4, 2, "bf16")) == 0  # no rows: nothing is launched


def test_binding_checks_sizes():
    packed = torch.empty(2, B.dynmo_mxfp4_bytes(5, 40), dtype=torch.uint8)
    assert B._mxfp4_sizes(torch.empty(2, 5, 40, dtype=torch.float32), packed) == (2, 5, 40, 0)
    assert B._mxfp4_sizes(torch.empty(5, 40, dtype=torch.bfloat16), packed[0]) == (1, 5, 40, 1)
    for rows, K in ((1, 8), (16, 128), (17, 136), (100, 512), (33, 1032)):
        assert B._mxfp4_sizes(torch.empty(rows, K, dtype=torch.float32), torch.empty(B.dynmo_mxfp4_bytes(rows, K), dtype=torch.uint8)) == (1, rows, K, 0)
    for values, p in ((torch.empty(2, 5, 40, dtype=torch.float32), packed[0]), (torch.empty(2, 5, 40, dtype=torch.float32).half(), packed), (torch.empty(40, dtype=torch.float32), packed),
                      (torch.empty(2, 5, 40, dtype=torch.float32), packed.float())):
        with pytest.raises(ValueError):
            B._mxfp4_sizes(values, p)
    with pytest.raises(ValueError):  # not on the GPU
        B.dynmo_mxfp4_quantize(torch.empty(2, 5, 40, dtype=torch.float32), packed)


# ---- quantisation on the GPU --------------------------------------------------------------------------------------------------

def pack_ref(x):
    out = []
    for m in x:
        _, code, scale = orc.mxfp4_quantize(m)
        out.append(orc.mxfp4_pack(code, scale))
    return np.stack(out)


def awkward(shape, dtype, rng):
    """Values over the whole range of exponents, exact midpoints, zeros of both signs, subnormals, blocks of zeros."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-20, 20, size=shape[:-1] + (1,))
    x.reshape(-1)[::7] = 0.0
    x.reshape(-1)[3::11] *= -0.0
    mids = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0], size=shape)
    x[..., 1::3, :] = (mids * rng.choice([-1, 1], size=shape))[..., 1::3, :]
    x[..., 2::9, : shape[-1] // 2] = 0.0
    if shape[-2] > 4:
        x[..., 3, :] = 2.0 ** rng.integers(-149, -120, size=shape[-1])
        x[..., 4, :] = 2.0 ** 127 * (1 + rng.random(shape[-1]) * 0.99)
    t = torch.from_numpy(x.astype(np.float32))
    return t.bfloat16() if dtype == "bf16" else t


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,K", [(1, 1, 8), (1, 1, 32), (2, 5, 40), (1, 16, 128), (3, 17, 136), (1, 33, 520), (2, 100, 512), (1, 15, 1032),
                                      (1, 48, 2056), (5, 1, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize(n, rows, K, dtype):
    if dtype == "bf16" and K % 8:
        pytest.skip("refused")
    src = awkward((n, rows, K), dtype, np.random.default_rng(rows * 7 + K))
    x = src.float().numpy()
    packed = torch.full((n, B.dynmo_mxfp4_bytes(rows, K)), 0xA5, dtype=torch.uint8, device="cuda")
    B.dynmo_mxfp4_quantize(src.cuda(), packed)
    assert np.array_equal(packed.cpu().numpy(), pack_ref(x))
    values = torch.full_like(src, 7.0, device="cuda")
    B.dynmo_mxfp4_dequantize(packed, values)
    assert np.array_equal(values.float().cpu().numpy().astype(np.float64), orc.mxfp4_quantize(x)[0])
    other = torch.empty((n, rows, (K + 7) // 8 * 8), dtype=torch.float32 if dtype == "bf16" else torch.bfloat16, device="cuda")
    if other.shape[-1] == K:  # the other type holds the same values
        B.dynmo_mxfp4_dequantize(packed, other)
        assert torch.equal(other.float(), values.float())
    again = torch.zeros_like(packed)
    B.dynmo_mxfp4_quantize(values, again)
    back = torch.empty_like(values)
    B.dynmo_mxfp4_dequantize(again, back)
    assert torch.equal(back, values)


@pytest.mark.gpu
def test_quantize_infinities_and_nan():
    x = np.random.default_rng(1).standard_normal((20, 96)).astype(np.float32)
    x[3, 5], x[4, 40], x[5, 95], x[6, 0] = np.inf, -np.inf, np.nan, np.finfo(np.float32).max
    for src in (torch.from_numpy(x), bf16(x)):
        packed = torch.empty(B.dynmo_mxfp4_bytes(20, 96), dtype=torch.uint8, device="cuda")
        B.dynmo_mxfp4_quantize(src.cuda(), packed)
        assert np.array_equal(packed.cpu().numpy(), pack_ref(src.float().numpy()[None])[0])
        values = torch.empty_like(src, device="cuda")
        B.dynmo_mxfp4_dequantize(packed, values)
        np.testing.assert_array_equal(values.float().cpu().numpy(), orc.mxfp4_quantize(src.float().numpy())[0].astype(np.float32))


# ---- the FFN on the GPU -----------------------------------------------------------------------------------------------------

def make_weights(E, H, F, rng):
    """Packed weights on the GPU and the values they stand for."""
    packed, values = [], []
    for rows, K in ((F, H), (F, H), (H, F)):
        w = torch.from_numpy((rng.standard_normal((E, rows, K)) / np.sqrt(K)).astype(np.float32)).cuda()
        p = torch.empty((E, B.dynmo_mxfp4_bytes(rows, K)), dtype=torch.uint8, device="cuda")
        B.dynmo_mxfp4_quantize(w, p)
        v = torch.empty_like(w)
        B.dynmo_mxfp4_dequantize(p, v)
        packed.append(p)
        values.append(v.cpu().numpy().astype(np.float64))
    return packed, values


def tolerances(x_p, seg, W, ref):
    """|dG|, |dU| and |dY| (before its rounding) as derived above."""
    Y, G, U, A = ref
    xq = np.abs(orc.mxfp4_quantize(x_p)[0])
    steps = lambda K: (-(-K // 128) + 2) * 2.0 ** -23  # noqa: E731
    dG, dU, dY = np.zeros_like(G), np.zeros_like(U), np.zeros_like(Y)
    for e in range(len(W[0])):
        rows = slice(int(seg[e]), int(seg[e + 1]))
        dG[rows] = steps(x_p.shape[1]) * (xq[rows] @ np.abs(W[0][e]).T)
        dU[rows] = steps(x_p.shape[1]) * (xq[rows] @ np.abs(W[1][e]).T)
    silu = np.abs(G * orc._sigmoid(G))
    dA = 1.1 * dG * np.abs(U) + silu * dU + (8 + 8 * np.abs(G)) * 2.0 ** -24 * np.abs(A)
    mid, _, _ = orc.mxfp4_quantize(A)
    high, _, s_high = orc.mxfp4_quantize(np.sign(A) * (np.abs(A) + dA))
    low, _, s_low = orc.mxfp4_quantize(np.sign(A) * np.maximum(np.abs(A) - dA, 0))
    F = A.shape[1]
    unit = np.repeat(2.0 ** (s_high.astype(np.float64) - 127), 32, axis=-1)[:, :F]
    moved = np.repeat(s_high != s_low, 32, axis=-1)[:, :F]
    slack = np.maximum(np.abs(high - mid), np.abs(low - mid)) + np.where(moved, 2 * unit, 0)
    for e in range(len(W[0])):
        rows = slice(int(seg[e]), int(seg[e + 1]))
        dY[rows] = (slack[rows] + steps(F) * (np.abs(mid[rows]) + slack[rows])) @ np.abs(W[2][e]).T
    return dG, dU, dY


def segments(counts, T, k, rng):
    """src_slot and seg_offsets with these many rows per expert, slots drawn without order."""
    R = int(sum(counts))
    slots = rng.permutation(T * k)[:R].astype(np.int32)
    return slots, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def check_ffn(T, H, F, E, k, counts, gather, save=False, seed=0, sigma=1.0):
    rng = np.random.default_rng(seed + T * 31 + H + F * 7 + E)
    R = int(sum(counts))
    assert len(counts) == E and R <= T * k
    packed, W = make_weights(E, H, F, rng)
    x = bf16(sigma * rng.standard_normal((T if gather else T * k, H)))
    slots, seg = segments(counts, T, k, rng)
    d = B.make_desc(T, H, F, E, k, "bf16")
    y = torch.full((T * k, H), 7.0, dtype=torch.bfloat16, device="cuda")
    G, U = (torch.full((T * k, F), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)) if save else (None, None)
    ws = torch.full((B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    full = np.concatenate([slots, np.full(T * k - R, -1, np.int32)])
    B.dynmo_grouped_ffn_mxfp4(d, x.cuda(), torch.from_numpy(full).cuda() if gather else None, torch.from_numpy(seg).cuda(), *packed, y, G, U, ws)
    x_p = x.float().numpy()[slots // k] if gather else x.float().numpy()[:R]
    ref = orc.grouped_ffn_mxfp4(x_p, seg, *W)
    dG, dU, dY = tolerances(x_p, seg, W, ref)
    got = y.float().cpu().numpy().astype(np.float64)
    assert (got[R:] == 7.0).all()  # rows behind the last segment are left as they were
    over = np.abs(got[:R] - ref[0]) - dY * (1 + BF16) - BF16 * np.abs(ref[0])
    assert (over <= 1e-30).all(), over.max()
    if save:
        for t, r, dr in ((G, ref[1], dG), (U, ref[2], dU)):
            g = t.float().cpu().numpy().astype(np.float64)
            assert (g[R:] == 7.0).all() and (np.abs(g[:R] - r) <= dr * (1 + BF16) + BF16 * np.abs(r) + 1e-30).all()
    return y


FFN_CASES = [
    (1, 8, 8, 1, 1, [1]), (1, 128, 256, 4, 2, [1, 0, 0, 1]), (3, 136, 72, 2, 2, [6, 0]), (5, 520, 520, 3, 3, [0, 15, 0]),
    (17, 1032, 264, 2, 1, [16, 1]), (40, 256, 640, 4, 2, [33, 0, 30, 17]), (150, 264, 136, 3, 2, [128, 129, 43]),
    (130, 2056, 520, 2, 2, [257, 3]), (70, 512, 1032, 64, 8, [9] * 62 + [0, 2]), (300, 392, 304, 5, 1, [0, 300, 0, 0, 0]),
    (600, 128, 128, 1, 1, [577]),
    # experts that took more rows than there are tokens (a token may name one twice)
    (16, 264, 136, 4, 4, [40, 0, 3, 20]), (64, 520, 264, 5, 4, [130, 0, 70, 0, 56]), (33, 1544, 1096, 2, 2, [50, 16])]


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,F,E,k,counts", FFN_CASES)
@pytest.mark.parametrize("gather", [False, True])
def test_ffn(T, H, F, E, k, counts, gather):
    check_ffn(T, H, F, E, k, counts, gather, save=gather)


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,F,E,counts,save", [(10700, 1032, 8200, 2, [300, 37], False), (52480, 1032, 264, 3, [130, 0, 257], False),
                                                  (16000, 1032, 2056, 2, [17, 200], True)])
def test_ffn_wide_tiles(T, H, F, E, counts, save):
    """Sizes that take tiles of 256 weight rows (chosen by the rows there may be; few are routed here): gate/up and a down product with a long
    sum, down by the number of its tiles, gate/up alone with G and U saved."""
    check_ffn(T, H, F, E, 1, counts, True, save=save)


@pytest.mark.gpu
def test_ffn_workspace_at_any_address_and_nothing_written_behind_it():
    T, H, F, E, k = 20, 264, 136, 3, 2
    rng = np.random.default_rng(5)
    packed, _ = make_weights(E, H, F, rng)
    x = bf16(rng.standard_normal((T * k, H))).cuda()
    d = B.make_desc(T, H, F, E, k, "bf16")
    seg = torch.tensor([0, 17, 18, 40], dtype=torch.int32, device="cuda")
    n = B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d)
    out = []
    for at in (0, 1, 255):
        ws = torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        y = torch.empty((T * k, H), dtype=torch.bfloat16, device="cuda")
        B.dynmo_grouped_ffn_mxfp4(d, x, None, seg, *packed, y, None, None, ws[at:at + n])
        assert (ws[:at] == 0x5A).all() and (ws[at + n:] == 0x5A).all()
        out.append(y)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


@pytest.mark.gpu
def test_ffn_no_rows_at_all():
    check_ffn(4, 64, 64, 3, 2, [0, 0, 0], True)


@pytest.mark.gpu
@pytest.mark.parametrize("sigma", [1e-30, 1e-3, 1e3])
def test_ffn_sizes_of_values(sigma):
    check_ffn(20, 256, 256, 2, 1, [11, 9], False, sigma=sigma)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 200])
def test_ffn_rows_of_nan_stay_alone(T):
    rng = np.random.default_rng(4)
    packed, W = make_weights(2, 128, 192, rng)
    x = rng.standard_normal((T, 128)).astype(np.float32)
    bad = x.copy()
    bad[1, 5], bad[4, 100] = np.nan, np.inf
    d = B.make_desc(T, 128, 192, 2, 1, "bf16")
    seg = torch.tensor([0, 3, T], dtype=torch.int32, device="cuda")
    ws = torch.full((B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    out = []
    for v in (x, bad):
        y = torch.empty((T, 128), dtype=torch.bfloat16, device="cuda")
        B.dynmo_grouped_ffn_mxfp4(d, bf16(v).cuda(), None, seg, *packed, y, None, None, ws)
        out.append(y.float().cpu().numpy())
    rows = np.ones(T, bool)
    rows[[1, 4]] = False
    assert np.isnan(out[1][~rows]).all() and np.array_equal(out[0][rows], out[1][rows]) and np.isfinite(out[0]).all()


@pytest.mark.gpu
def test_layer_run_together_and_its_gradient():
    """Scored routing, permutation, 4-bit experts and combine as a layer runs them, with the straight-through backward pass."""
    T, H, F, E, k = 90, 128, 160, 8, 3
    rng = np.random.default_rng(12)
    packed, W = make_weights(E, H, F, rng)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    logits[:, 3] = -np.inf
    logits[5], logits[6, 4:] = -np.inf, -np.inf  # a token without an expert, one with three of four groups' experts left
    x, dout = bf16(rng.standard_normal((T, H))), bf16(rng.standard_normal((T, H)))
    rule = dict(score="sigmoid", groups=4, top_groups=2, group_best=2, renormalize=True, scale=2.0)
    layer = RoutedFFNLayer(T, H, F, E, k, "bf16")
    lg = torch.from_numpy(logits).cuda()
    layer.route_scored(lg, B.make_rule(**rule), torch.from_numpy(bias).cuda())
    idx, gate = orc.route_scored(logits, bias, k, **rule)
    assert np.array_equal(layer.expert_idx.cpu().numpy(), idx)
    served = layer.forward_mxfp4(x.cuda(), *packed, out=torch.empty((T, H), dtype=torch.bfloat16, device="cuda"))
    out = layer.forward_mxfp4(x.cuda(), *packed, train=True)
    assert torch.equal(served, out)
    x_p, seg, src, dst = orc.permute(x.float().numpy(), idx, E)[:4]
    R = int(seg[-1])
    assert R < T * k and layer.seg_offsets.cpu().numpy().tolist() == list(seg)
    ref = orc.grouped_ffn_mxfp4(x_p[:R], seg, *W)
    dG, dU, dY = tolerances(x_p[:R], seg, W, ref)
    y = np.concatenate([ref[0], np.zeros((T * k - R, H))])
    tol = np.concatenate([dY * (1 + BF16) + BF16 * np.abs(ref[0]), np.zeros((T * k - R, H))])
    want, slack = orc.combine(y, dst, gate, None, T), orc.combine(tol, dst, np.abs(gate), None, T)
    size = orc.combine(np.abs(y), dst, np.abs(gate), None, T)
    got = out.float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= slack * (1 + BF16) + BF16 * np.abs(want) + 64 * 2.0 ** -24 * size).all()
    assert (got[5] == 0).all()
    # straight through: the gradient of the FFN with the dequantised weights at the saved G, U
    Wd = [torch.from_numpy(w).bfloat16().cuda() for w in W]
    dx = layer.backward(dout.cuda(), *Wd)
    dl = layer.route_bwd(lg)
    do = dout.float().numpy()
    y_gpu = layer.y_p.float().cpu().numpy()
    dy_p, dgate = orc.combine_bwd(do, y_gpu, dst, layer.gate_w.cpu().numpy())
    Gs, Us = layer.G.float().cpu().numpy()[:R], layer.U.float().cpu().numpy()[:R]
    bwd = orc.grouped_ffn_bwd(dy_p[:R], x_p[:R], Gs, Us, seg, *W)
    dx_ref = orc.permute_bwd(np.concatenate([bwd[0], np.zeros((T * k - R, H))]), dst, None)
    # dy_p, dA, dG, dU and dx_p are rounded to bf16 on the way, dx once more: five half steps of values that the products sum with random signs
    err = np.abs(dx.float().cpu().numpy() - dx_ref).max() / np.abs(dx_ref).max()
    assert err <= 5 * BF16
    ref_dl = orc.route_scored_bwd(dgate, logits, idx, "sigmoid", True, 2.0)
    assert np.abs(dl.cpu().numpy() - ref_dl).max() <= 2.0 ** -12 * np.abs(ref_dl).max()  # dgate: a dot product of 128 terms in fp32


@pytest.mark.gpu
def test_ffn_captured_with_two_workspaces():
    T, H, F, E, k = 64, 256, 256, 4, 2
    rng = np.random.default_rng(6)
    packed, W = make_weights(E, H, F, rng)
    d = B.make_desc(T, H, F, E, k, "bf16")
    seg = torch.tensor([0, 40, 40, 100, 128], dtype=torch.int32, device="cuda")
    xs = [torch.empty((T * k, H), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ys = [torch.zeros((T * k, H), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    wss = [torch.empty(B.dynmo_grouped_ffn_mxfp4_workspace_bytes(d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        B.dynmo_grouped_ffn_mxfp4(d, xs[0], None, seg, *packed, ys[0], None, None, wss[0])
        with torch.cuda.stream(side):
            B.dynmo_grouped_ffn_mxfp4(d, xs[1], None, seg, *packed, ys[1], None, None, wss[1])
        main.wait_stream(side)
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in xs:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(xs, ys):
            eager = torch.empty_like(y)
            ws = torch.empty_like(wss[0])
            B.dynmo_grouped_ffn_mxfp4(d, x, None, seg, *packed, eager, None, None, ws)
            assert torch.equal(eager, y)


def test_every_profiled_role_has_a_name():
    names = [B.dynmo_profile_kernel_name(i) for i in range(B.dynmo_profile_kernel_count())]
    assert len(set(names)) == len(names) and names[-2:] == ["mxfp4_quantize", "mxfp4_dequantize"]


@pytest.mark.gpu
def test_profiling_sees_the_calls():
    T, H, F, E, k = 40, 256, 256, 4, 2
    rng = np.random.default_rng(8)
    packed, _ = make_weights(E, H, F, rng)
    layer = RoutedFFNLayer(T, H, F, E, k, "bf16")
    B.dynmo_profile_reset()
    B.dynmo_profile_enable(True)
    try:
        layer.route_scored(torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda(), B.make_rule("sigmoid"))
        layer.forward_mxfp4(bf16(rng.standard_normal((T, H))).cuda(), *packed)
    finally:
        B.dynmo_profile_enable(False)
    got = {B.dynmo_profile_kernel_name(i): B.dynmo_profile_read(i) for i in range(B.dynmo_profile_kernel_count())}
    B.dynmo_profile_reset()
    for name in ("route_topk", "mxfp4_quantize", "ffn_gateup", "ffn_down", "combine"):
        assert got[name][1] == 1 and got[name][0] > 0, name
