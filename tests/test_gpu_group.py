"""Group-scaled rows on the GPU against plain 64-bit arithmetic.

Tolerances, derived from the arithmetic: whole numbers and scales are exact.  A product's sum runs in
32-bit floats, at most K/32 + 64 additions and roundings deep (32 products to a step, then one step
after another), each off by at most 2^-24 of the sum of magnitudes S, in which a weight counts as its
unsigned field plus its zero point (8 when signed); the result is rounded once to its type, by at most
eps/2 of its value.  Input gradients of 16-bit types round each weight to bf16 once more (2^-8 of
|dy| |w|) or keep 16 bits of it."""
import numpy as np
import pytest
import torch

import paper_1809_10572_amd as samd
from paper_1809_10572_amd import GroupRows
import group_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def half_step(typ):
    return torch.finfo(TYPES[typ]).eps / 2


def rng_rows(rng, rows, cols, group, signed):
    """Random 4-bit rows: (GroupRows on the GPU, float64 values, float64 magnitudes s * (field + zero))."""
    q = rng.integers(0, 16, (rows, cols), dtype=np.uint32)
    per = -(-cols // 8)
    wide = np.zeros((rows, per * 8), dtype=np.uint32)
    wide[:, :cols] = q
    words = np.zeros((rows, per), dtype=np.uint32)
    for i in range(8):
        words |= wide[:, i::8] << np.uint32(4 * i)
    groups = -(-cols // group)
    scale = (rng.random((rows, groups)) + 0.5).astype(np.float32) / np.float32(4 * np.sqrt(cols))
    zero = None if signed else rng.integers(0, 16, (rows, groups), dtype=np.uint8)
    whole = q.astype(np.int64)
    if signed:
        whole = np.where(whole >= 8, whole - 16, whole)
    at = np.arange(cols) // group
    fields = (q ^ 8 if signed else q).astype(np.int64) + (8 if signed else zero.astype(np.int64)[:, at])
    r = GroupRows(torch.from_numpy(words.view(np.int32)).to(DEV), torch.from_numpy(scale).to(DEV),
                  None if signed else torch.from_numpy(zero).to(DEV), cols, 4, group)
    return r, ref.values(whole, scale, zero, group), scale.astype(np.float64)[:, at] * fields


def rng_matrix(rng, rows, cols, typ, pad=0):
    """A float matrix on the GPU (with `pad` columns of NaN behind every row) and its float64 values."""
    t = torch.from_numpy(rng.standard_normal((rows, cols + pad)).astype(np.float32)).to(TYPES[typ])
    if pad:
        t[:, cols:] = float("nan")
    t = t.to(DEV)[:, :cols]
    return t, f64(t)


def close(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape
    off = np.abs(got - want) - bound
    fine = bool(np.isfinite(got).all() and (off <= 0).all())
    assert fine, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def depth(n):
    return (n / 32 + 64) * 2.0 ** -24


# ---- quantisation ---------------------------------------------------------------------------------

QUANT = [(1, 1), (3, 7), (2, 8), (5, 31), (4, 32), (3, 33), (7, 129), (2, 515), (33, 1000), (1, 4099)]


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize_follows_the_rule(typ, bits, signed, group):
    rng = np.random.default_rng(bits + group + signed)
    for rows, cols in QUANT:
        for pad in (0, 3, 8):
            x, _ = rng_matrix(rng, rows, cols, typ, pad)
            if cols > 40:
                x[0, 32:40] = 0
            r = samd.group_quantize(x, bits, signed, group)
            q, scale, zero = ref.quantize(x.cpu().float().numpy(), bits, signed, group)
            words = r.q.cpu().numpy()
            assert words.shape == (rows, samd.row_words(cols, bits))
            assert np.array_equal(ref.unpack(words, cols, bits, signed), q), (rows, cols, pad)
            assert not ref.spare_bits(words, cols, bits).any()
            assert np.array_equal(r.scale.cpu().numpy(), scale)
            assert zero is None and r.zero is None or np.array_equal(r.zero.cpu().numpy(), zero)
            # and back, rounded once to the type
            back = samd.group_dequantize(r, TYPES[typ])
            exact = torch.from_numpy(ref.values(q, scale, zero, group).astype(np.float32)).to(TYPES[typ])
            assert torch.equal(back.cpu(), exact)


@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("bits", [4, 8])
def test_quantize_of_unusual_groups(bits, signed):
    x = torch.zeros(10, 96, dtype=torch.float32)
    x[1, 3] = float("nan")
    x[2, 40] = float("inf")
    x[3, 95] = float("-inf")
    x[4] = 2.0 ** -101
    x[5, 7] = 2.0 ** -100
    x[6, :32] = 3.0e38
    x[6, 5] = -3.0e38          # a span beyond the largest float where both signs count
    x[7] = -1.5
    x[8] = 2.5
    x[9] = torch.arange(96) - 40.0
    r = samd.group_quantize(x.to(DEV), bits, signed, 32)
    q, scale, zero = ref.quantize(x.numpy(), bits, signed, 32)
    assert np.array_equal(ref.unpack(r.q.cpu().numpy(), 96, bits, signed), q)
    assert np.array_equal(r.scale.cpu().numpy(), scale, equal_nan=True)
    assert signed or np.array_equal(r.zero.cpu().numpy(), zero)
    back = samd.group_dequantize(r, torch.float32).cpu().numpy()
    nan = np.isnan(back)
    assert nan[1, :32].all() and nan[2, 32:64].all() and nan[3, 64:].all() and nan[6, :32].all() == (not signed)
    assert nan.sum() == 96 + (0 if signed else 32)
    assert not back[4].any() and not back[0].any()


def test_rows_pass_through_pack_and_unpack():
    x = torch.randn(6, 70, device=DEV)
    for bits in (4, 8):
        for signed in (True, False):
            r = samd.group_quantize(x, bits, signed, 32)
            v = samd.unpack(r.q, 70, bits, signed)
            assert torch.equal(samd.pack(v, bits, signed), r.q)


def test_dequantize_writes_its_rows_only():
    r = samd.group_quantize(torch.randn(5, 45, device=DEV), 8, True, 32)
    buf = torch.full((7, 60), 7.0, device=DEV, dtype=torch.float16)
    samd.group_dequantize(r, out=buf[1:6, 2:47])
    want = samd.group_dequantize(r, torch.float16)
    assert torch.equal(buf[1:6, 2:47], want)
    buf[1:6, 2:47] = 7.0
    assert (buf == 7.0).all()


# ---- products -------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 3, 31), (1, 33, 8), (1, 70, 257), (2, 64, 4096), (3, 37, 130), (4, 40, 2051), (5, 129, 513),
         (8, 16, 64), (15, 31, 97), (16, 96, 1024), (17, 257, 640), (33, 48, 4100), (64, 160, 256), (65, 130, 72), (100, 64, 2304),
         (128, 128, 128), (131, 301, 1000), (260, 513, 264)]


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("size", SIZES)
def test_matmul(typ, signed, size):
    T, M, K = size
    rng = np.random.default_rng(T + M + K)
    for group, pad in ((32, 0), (64, 5), (128, 8)):
        w, values, sizes = rng_rows(rng, M, K, group, signed)
        x, xv = rng_matrix(rng, T, K, typ, pad)
        y = samd.group_matmul(x, w)
        assert y.dtype == x.dtype
        want = xv @ values.T
        close(y, want, half_step(typ) * np.abs(want) + depth(K) * (np.abs(xv) @ sizes.T), (group, pad))


def test_matmul_of_the_largest_words_and_empty_rows():
    """Every field at its extreme, and tokens of zeros: exact results."""
    for typ in TYPES:
        for T in (1, 3, 20, 130):
            M, K = 48, 160
            q = torch.full((M, K // 8), -1, dtype=torch.int32, device=DEV)        # fields 15: 15 unsigned, -1 signed
            q[M // 2:] = -2004318072                                             # fields 8: 8 unsigned, -8 signed
            scale = torch.ones(M, K // 32, device=DEV)
            x = torch.ones(T, K, device=DEV, dtype=TYPES[typ])
            x[T // 2] = 0
            zero = torch.full((M, K // 32), 15, dtype=torch.uint8, device=DEV)
            for z, low, high in ((None, -1, -8), (zero, 0, -7)):
                y = samd.group_matmul(x, GroupRows(q, scale, z, K, 4, 32)).float()
                want = torch.empty(T, M, device=DEV)
                want[:, :M // 2], want[:, M // 2:] = low * K, high * K
                want[T // 2] = 0
                assert torch.equal(y, want.to(TYPES[typ]).float()), (typ, T, z is None)


@pytest.mark.parametrize("T", [2, 20, 140])
def test_matmul_keeps_infinities_in_their_row(T):
    rng = np.random.default_rng(5)
    w, values, _ = rng_rows(rng, 40, 200, 64, False)
    for typ in TYPES:
        x, _ = rng_matrix(rng, T, 200, typ)
        clean = samd.group_matmul(x, w)
        x[0, 17], x[1, 199] = float("inf"), float("nan")
        y = samd.group_matmul(x, w)
        assert not torch.isfinite(y[0]).any() and torch.isnan(y[1]).all()
        assert torch.equal(y[2:], clean[2:])


@pytest.mark.parametrize("T", [1, 3, 18, 70, 200])
def test_results_stay_inside_their_rows(T):
    """Padded outputs keep what lies between and behind their rows; whatever lies between input rows
    (NaN here) is never read."""
    rng = np.random.default_rng(T)
    M, K = 50, 90
    w, values, _ = rng_rows(rng, M, K, 32, True)
    for typ in TYPES:
        x, xv = rng_matrix(rng, T, K, typ, 6)
        dy, dyv = rng_matrix(rng, T, M, typ, 3)
        buf = torch.full((T + 2, M + 9), 3.0, device=DEV, dtype=TYPES[typ])
        samd.group_matmul(x, w, out=buf[1:T + 1, 4:M + 4])
        assert torch.equal(buf[1:T + 1, 4:M + 4], samd.group_matmul(x.contiguous(), w))
        buf[1:T + 1, 4:M + 4] = 3.0
        assert (buf == 3.0).all()
        samd.group_gated(x, w, w, out=buf[1:T + 1, 4:M + 4])
        buf[1:T + 1, 4:M + 4] = 3.0
        assert (buf == 3.0).all()
        buf = torch.full((T + 2, K + 9), 3.0, device=DEV, dtype=TYPES[typ])
        samd.group_matmul_grad(dy, w, out=buf[1:T + 1, 4:K + 4])
        assert torch.equal(buf[1:T + 1, 4:K + 4], samd.group_matmul_grad(dy.contiguous(), w))
        buf[1:T + 1, 4:K + 4] = 3.0
        assert (buf == 3.0).all()


def test_words_and_scales_at_any_word():
    """Weights that start 4, 8 and 12 bytes behind a 16-byte boundary, activations at any element."""
    rng = np.random.default_rng(9)
    for K in (256, 1024):
        for T in (1, 2, 16, 80):
            w, _, _ = rng_rows(rng, 32, K, 32, False)
            x, _ = rng_matrix(rng, T, K, "bf16")
            dy, _ = rng_matrix(rng, T, 32, "bf16")
            y, dx = samd.group_matmul(x, w), samd.group_matmul_grad(dy, w)
            for off in (1, 2, 3):
                def moved(t):
                    m = torch.empty(t.numel() + off, dtype=t.dtype, device=DEV)[off:]
                    return m.copy_(t.flatten()).view(t.shape)
                v = GroupRows(moved(w.q), moved(w.scale), moved(w.zero), K, 4, 32)
                assert torch.equal(samd.group_matmul(moved(x), v), y)
                assert torch.equal(samd.group_matmul_grad(moved(dy), v), dx)


# ---- input gradients ------------------------------------------------------------------------------

def grad_bound(typ, want, dyv, values, sizes):
    rounding = {"f32": 0.0, "f16": 2.0 ** -15, "bf16": 2.0 ** -8}[typ]
    return half_step(typ) * np.abs(want) + rounding * (np.abs(dyv) @ np.abs(values)) + depth(values.shape[0]) * (np.abs(dyv) @ sizes)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("size", SIZES)
def test_matmul_grad(typ, signed, size):
    T, M, K = size
    rng = np.random.default_rng(T + M + K + 1)
    for group, pad in ((32, 0), (64, 5), (128, 8)):
        w, values, sizes = rng_rows(rng, M, K, group, signed)
        w2, values2, sizes2 = rng_rows(rng, M, K, group, signed)
        dy, dyv = rng_matrix(rng, T, M, typ, pad)
        dy2, dyv2 = rng_matrix(rng, T, M, typ, pad)
        want = dyv @ values
        close(samd.group_matmul_grad(dy, w), want, grad_bound(typ, want, dyv, values, sizes), (group, pad))
        both = want + dyv2 @ values2
        bound = grad_bound(typ, both, np.hstack((dyv, dyv2)), np.vstack((values, values2)), np.vstack((sizes, sizes2)))
        close(samd.group_matmul_grad(dy, w, dy2, w2), both, bound, (group, pad, "two"))


@pytest.mark.parametrize("size", [(3, 50, 70), (40, 96, 200), (150, 260, 300)])
def test_gradient_is_the_transpose_of_the_product(size):
    """<y, W x> = <W^T y, x>: the product is linear, so this is its derivative by differences."""
    T, M, K = size
    rng = np.random.default_rng(T)
    w, values, sizes = rng_rows(rng, M, K, 32, False)
    x, xv = rng_matrix(rng, T, K, "f32")
    dy, dyv = rng_matrix(rng, T, M, "f32")
    left = (dyv * f64(samd.group_matmul(x, w))).sum()
    right = (f64(samd.group_matmul_grad(dy, w)) * xv).sum()
    total = (np.abs(dyv) * (np.abs(xv) @ sizes.T)).sum()
    assert abs(left - right) <= (depth(K) + depth(M) + 2 * 2.0 ** -24) * total


# ---- the gated block ------------------------------------------------------------------------------

@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES)
def test_gated(typ, act, size):
    T, M, K = size
    rng = np.random.default_rng(T + M + K + 2)
    for group, signed, pad in ((32, True, 0), (64, False, 5), (128, True, 8)):
        wg, gv, gs = rng_rows(rng, M, K, group, signed)
        wu, uv, us = rng_rows(rng, M, K, group, signed)
        x, xv = rng_matrix(rng, T, K, typ, pad)
        g, u = xv @ gv.T, xv @ uv.T
        dg, du = depth(K) * (np.abs(xv) @ gs.T), depth(K) * (np.abs(xv) @ us.T)
        a, _ = ref.activation(g, act)
        want = a * u
        # |act'| <= 1.2; act and its product take 16 units in the last 32-bit place
        bound = half_step(typ) * np.abs(want) + 1.2 * dg * (np.abs(u) + du) + np.abs(a) * du + 16 * 2.0 ** -24 * np.abs(g * u)
        close(samd.group_gated(x, wg, wu, act), want, bound, (group, signed))
        h, g8, u8 = samd.group_gated_save(x, wg, wu, act)
        close(h, want, bound, (group, signed, "save"))
        for r, v, d in ((g8, g, dg), (u8, u, du)):
            assert (r.bits, r.group, r.cols, r.zero) == (8, samd.GATED_GROUP, M, None)
            q = ref.unpack(r.q.cpu().numpy().reshape(T, -1), M, 8, True)
            assert np.abs(q).max() <= 127 and not ref.spare_bits(r.q.cpu().numpy().reshape(T, -1), M, 8).any()
            scale = r.scale.cpu().numpy().reshape(T, -1).astype(np.float64)
            at = np.arange(M) // 32
            # half a step of the scale, and the sums' own error, also in the group's largest value
            span = np.maximum.reduceat(d, np.arange(0, M, 32), axis=1)[:, at]
            off = np.abs(scale[:, at] * q - v) - (0.5 * scale[:, at] * (1 + 2.0 ** -20) + d + span + 2.0 ** -22 * np.abs(v))
            assert (off <= 0).all(), off.max()
            big = np.maximum.reduceat(np.abs(v), np.arange(0, M, 32), axis=1)
            assert (np.abs(scale * 127 - big) <= np.maximum.reduceat(d, np.arange(0, M, 32), axis=1) + 2.0 ** -22 * big).all()


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_grad(typ, act):
    for T, M, group, pad in ((1, 1, 32, 0), (3, 7, 64, 1), (5, 33, 32, 3), (4, 128, 128, 8), (17, 515, 32, 0), (64, 96, 64, 8)):
        rng = np.random.default_rng(T + M)
        dh, dhv = rng_matrix(rng, T, M, typ, pad)
        spread = np.exp(rng.uniform(-3, 3, (T, 1))).astype(np.float32)   # slopes near 0, 1 and between
        g = samd.group_quantize(torch.from_numpy(spread * rng.standard_normal((T, M)).astype(np.float32)).to(DEV), 8, True, group)
        u = samd.group_quantize(torch.from_numpy(rng.standard_normal((T, M)).astype(np.float32)).to(DEV), 8, True, group)
        gv, uv = f64(samd.group_dequantize(g)), f64(samd.group_dequantize(u))
        a, slope = ref.activation(gv, act)
        dg, du = samd.group_gated_grad(dh, g, u, act)
        # the 32-bit terms of act' are at most 1 + |g| each and off by 8 units in the last place
        err = 2.0 ** -21 * (1 + np.abs(gv))
        close(dg, dhv * uv * slope, half_step(typ) * np.abs(dhv * uv * slope) + err * np.abs(dhv * uv) + tiny(typ), "dg")
        close(du, dhv * a, half_step(typ) * np.abs(dhv * a) + err * np.abs(dhv * gv) + tiny(typ), "du")
        # the formula against differences, in 64 bits: an error of e^2 for a step of e
        e = 1e-5
        numeric = (ref.activation(gv + e, act)[0] - ref.activation(gv - e, act)[0]) / (2 * e)
        assert np.abs(numeric - slope).max() < 1e-8


def tiny(typ):
    """Half the smallest step of a type, for results below its normal range."""
    return {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}[typ]


# ---- many tokens: the larger tiles ----------------------------------------------------------------

def gpu_rows(gen, rows, cols, group, signed):
    """Random 4-bit rows made and read on the GPU: (GroupRows, float64 values, float64 magnitudes)."""
    q = torch.randint(0, 16, (rows, -(-cols // 8) * 8), generator=gen, device=DEV)
    q[:, cols:] = 0
    words = (q.view(rows, -1, 8) << torch.arange(0, 32, 4, device=DEV)).sum(2)
    words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
    groups = -(-cols // group)
    scale = (torch.rand(rows, groups, generator=gen, device=DEV) + 0.5) / (4 * cols ** 0.5)
    zero = None if signed else torch.randint(0, 16, (rows, groups), generator=gen, device=DEV).to(torch.uint8)
    at = torch.arange(cols, device=DEV) // group
    q = q[:, :cols]
    whole = torch.where(q >= 8, q - 16, q) if signed else q - zero.long()[:, at]
    fields = (q ^ 8) + 8 if signed else q + zero.long()[:, at]
    s = scale.double()[:, at]
    return GroupRows(words, scale, zero, cols, 4, group), s * whole, s * fields


def gpu_matrix(gen, rows, cols, typ, pad):
    t = torch.full((rows, cols + pad), float("nan"), device=DEV, dtype=TYPES[typ])[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=gen, device=DEV))
    return t, t.double()


def gpu_close(got, want, bound, what=""):
    off = (got.double() - want).abs() - bound
    fine = bool(torch.isfinite(got).all()) and float(off.max()) <= 0
    assert fine, (what, float(off.max()))


# tokens, rows of the result, summed values: sizes for which few tiles of 64 x 64 are not the least work, whose
# sums run over several turns of the pipeline, with and without a ragged end, at even and odd row strides
MANY = [(1000, 2100, 1096, 0), (1000, 2000, 1024, 8), (510, 2000, 1100, 0), (500, 2100, 1088, 2), (2040, 4090, 576, 0),
        (2048, 4096, 330, 0), (300, 1100, 700, 3)]


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", MANY)
def test_many_tokens(typ, size):
    T, M, K, pad = size
    gen = torch.Generator(device=DEV).manual_seed(T + M)
    for group, signed in ((32, False), (64, True), (128, False)):
        w, values, sizes = gpu_rows(gen, M, K, group, signed)
        x, xv = gpu_matrix(gen, T, K, typ, pad)
        want = xv @ values.t()
        gpu_close(samd.group_matmul(x, w), want, half_step(typ) * want.abs() + depth(K) * (xv.abs() @ sizes.t()), ("y", group))
        # the same sizes for the gradient: M summed over, K of them the result's columns
        w, values, sizes = gpu_rows(gen, K, M, group, signed)
        w2, values2, sizes2 = gpu_rows(gen, K, M, group, signed)
        dy, dyv = gpu_matrix(gen, T, K, typ, pad)
        dy2, dyv2 = gpu_matrix(gen, T, K, typ, pad)
        rounding = {"f32": 0.0, "f16": 2.0 ** -15, "bf16": 2.0 ** -8}[typ]
        want = dyv @ values
        bound = rounding * (dyv.abs() @ values.abs()) + depth(K) * (dyv.abs() @ sizes)
        gpu_close(samd.group_matmul_grad(dy, w), want, half_step(typ) * want.abs() + bound, ("dx", group))
        want = want + dyv2 @ values2
        bound = bound + rounding * (dyv2.abs() @ values2.abs()) + depth(2 * K) * (dyv.abs() @ sizes + dyv2.abs() @ sizes2)
        gpu_close(samd.group_matmul_grad(dy, w, dy2, w2), want, half_step(typ) * want.abs() + bound, ("dx, two", group))


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(1000, 1050, 1096, 0), (1000, 1000, 1024, 8), (2040, 2030, 576, 0), (300, 550, 700, 3)])
def test_gated_of_many_tokens(typ, size):
    T, M, K, pad = size
    gen = torch.Generator(device=DEV).manual_seed(T + M)
    for group, signed, act in ((32, False, "silu"), (64, True, "gelu"), (128, False, "silu")):
        wg, gv, gs = gpu_rows(gen, M, K, group, signed)
        wu, uv, us = gpu_rows(gen, M, K, group, signed)
        x, xv = gpu_matrix(gen, T, K, typ, pad)
        g, u = xv @ gv.t(), xv @ uv.t()
        dg, du = depth(K) * (xv.abs() @ gs.t()), depth(K) * (xv.abs() @ us.t())
        a = torch.nn.functional.silu(g) if act == "silu" else torch.nn.functional.gelu(g)
        want = a * u
        bound = half_step(typ) * want.abs() + 1.2 * dg * (u.abs() + du) + a.abs() * du + 16 * 2.0 ** -24 * (g * u).abs()
        gpu_close(samd.group_gated(x, wg, wu, act), want, bound, group)
        h, g8, u8 = samd.group_gated_save(x, wg, wu, act)
        gpu_close(h, want, bound, (group, "save"))
        for r, v, d in ((g8, g, dg), (u8, u, du)):   # half a step of the scale and the sums' own error, also in the span
            back = samd.group_dequantize(r)
            step = r.scale.double().repeat_interleave(32, 1)[:, :M]
            span = torch.nn.functional.pad(d, (0, -M % 32)).view(T, -1, 32).amax(2).repeat_interleave(32, 1)[:, :M]
            gpu_close(back, v, 0.5 * step * (1 + 2.0 ** -20) + d + span + 2.0 ** -22 * v.abs(), (group, "stored"))


# ---- the operators together -----------------------------------------------------------------------

@pytest.mark.parametrize("typ", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T", [1, 6, 96])
def test_feed_forward_block_together(typ, T):
    """Weights quantised, the block run, its projections stored, its gradient taken: against 64 bits, each
    operator from what the one before it gave."""
    rng = np.random.default_rng(T)
    K, M = 160, 352
    def weights(rows, cols):
        r = samd.group_quantize(torch.from_numpy((rng.standard_normal((rows, cols)) / np.sqrt(cols)).astype(np.float32)).to(DEV),
                                4, False, 32)
        return r, f64(samd.group_dequantize(r))
    (wg, gv), (wu, uv), (wd, dv) = weights(M, K), weights(M, K), weights(K, M)
    x, xv = rng_matrix(rng, T, K, typ)
    h, g, u = samd.group_gated_save(x, wg, wu)
    y = samd.group_matmul(h, wd)
    dy, dyv = rng_matrix(rng, T, K, typ)
    dh = samd.group_matmul_grad(dy, wd)
    dg, du = samd.group_gated_grad(dh, g, u)
    dx = samd.group_matmul_grad(dg, wg, du, wu)
    step = 8 * half_step(typ) + 1e-5

    def near(got, want):
        got = f64(got)
        assert np.linalg.norm(got - want) <= step * np.linalg.norm(want)

    a, _ = ref.activation(xv @ gv.T, "silu")
    near(h, a * (xv @ uv.T))
    near(y, f64(h) @ dv.T)
    near(dh, dyv @ dv)
    gs, us = f64(samd.group_dequantize(g)), f64(samd.group_dequantize(u))
    a, slope = ref.activation(gs, "silu")
    near(dg, f64(dh) * us * slope)
    near(du, f64(dh) * a)
    near(dx, f64(dg) @ gv + f64(du) @ uv)


def _block(x, dh, wg, wu, wd, out):
    h, g, u = samd.group_gated_save(x, wg, wu)
    y = samd.group_matmul(h, wd)
    dg, du = samd.group_gated_grad(dh, g, u)
    dx = samd.group_matmul_grad(dg, wg, du, wu)
    q = samd.group_quantize(x, 8, True, 32)
    r = samd.group_dequantize(q, x.dtype)
    for o, v in zip(out, (h, y, dx, r)):
        o.copy_(v)


@pytest.mark.parametrize("T", [1, 12, 100])
def test_captured_and_replayed(T):
    rng = np.random.default_rng(T)
    K, M = 256, 384
    wg, wu, wd = (rng_rows(rng, r, c, 64, True)[0] for r, c in ((M, K), (M, K), (K, M)))
    x, dh = rng_matrix(rng, T, K, "bf16")[0], rng_matrix(rng, T, M, "bf16")[0]
    shapes = ((T, M), (T, K), (T, K), (T, K))
    eager = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    graphed = [torch.empty(s, device=DEV, dtype=torch.bfloat16) for s in shapes]
    _block(x, dh, wg, wu, wd, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _block(x, dh, wg, wu, wd, graphed)
    for i in range(4):
        x.copy_(rng_matrix(rng, T, K, "bf16")[0])
        for o in graphed:
            o.zero_()
        graph.replay()
        _block(x, dh, wg, wu, wd, eager)
        torch.cuda.synchronize()
        for a, b in zip(eager, graphed):
            assert torch.equal(a, b), i


def test_two_streams_at_once():
    rng = np.random.default_rng(3)
    K, M, T = 512, 640, 40
    wg, wu, wd = (rng_rows(rng, r, c, 64, False)[0] for r, c in ((M, K), (M, K), (K, M)))
    x, dh = rng_matrix(rng, T, K, "f16")[0], rng_matrix(rng, T, M, "f16")[0]
    shapes = ((T, M), (T, K), (T, K), (T, K))
    want, *got = ([torch.empty(s, device=DEV, dtype=torch.float16) for s in shapes] for _ in range(3))
    _block(x, dh, wg, wu, wd, want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, out in zip(streams, got):
            with torch.cuda.stream(s):
                _block(x, dh, wg, wu, wd, out)
    torch.cuda.synchronize()
    for out in got:
        for a, b in zip(want, out):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T", [0, 1])
def test_empty_sizes(T):
    rng = np.random.default_rng(0)
    w = rng_rows(rng, 8, 32, 32, True)[0]
    none = GroupRows(torch.empty(0, 4, dtype=torch.int32, device=DEV), torch.empty(0, 1, device=DEV), None, 32, 4, 32)
    x = torch.zeros(T, 32, device=DEV)
    assert samd.group_matmul(x, none).shape == (T, 0)
    assert samd.group_gated(x, none, none).shape == (T, 0)
    assert samd.group_quantize(torch.empty(T, 0, device=DEV), 4, True, 32).q.shape == (T, 0)
    if T == 0:
        assert samd.group_matmul(x, w).shape == (0, 8)
        h, g, u = samd.group_gated_save(x, w, w)
        assert h.shape == (0, 8) and g.q.shape == (0, 2) and u.scale.shape == (0, 1)
        assert samd.group_matmul_grad(torch.empty(0, 8, device=DEV), w).shape == (0, 32)
        assert samd.group_gated_grad(h, g, u)[0].shape == (0, 8)
        assert samd.group_dequantize(samd.group_quantize(x, 8, True, 32)).shape == (0, 32)


# ---- offsets past 32 bits -------------------------------------------------------------------------

def test_rows_far_apart():
    """Row strides of more than 2^30 elements: the third row starts past 2^31."""
    rng = np.random.default_rng(1)
    far, K, M = (1 << 30) + 72, 136, 40
    buf = torch.empty(2 * far + 256, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(2 * far + 256, dtype=torch.bfloat16, device=DEV)
    w = rng_rows(rng, M, K, 32, False)[0]
    x, dy = rng_matrix(rng, 3, K, "bf16")[0], rng_matrix(rng, 3, M, "bf16")[0]
    bx, by = torch.as_strided(buf, (3, K), (far, 1)), torch.as_strided(out, (3, M), (far, 1))
    bx.copy_(x)
    assert torch.equal(samd.group_matmul(bx, w, out=by), samd.group_matmul(x, w))
    r, s = samd.group_quantize(bx, 8, True, 32), samd.group_quantize(x, 8, True, 32)
    assert torch.equal(r.q, s.q) and torch.equal(r.scale, s.scale)
    back = torch.as_strided(out, (3, K), (far, 1))
    assert torch.equal(samd.group_dequantize(r, out=back), samd.group_dequantize(s, torch.bfloat16))
    bdy, bdx = torch.as_strided(buf, (3, M), (far, 1)), torch.as_strided(out, (3, K), (far, 1))
    bdy.copy_(dy)
    assert torch.equal(samd.group_matmul_grad(bdy, w, out=bdx), samd.group_matmul_grad(dy, w))


def test_weights_of_more_than_2_31_words():
    """70000 rows of 262144 weights (2.3e9 words): chosen rows against a small tensor of them alone."""
    M, K = 70000, 262144
    q = torch.randint(-2 ** 31, 2 ** 31 - 1, (1000, K // 8), dtype=torch.int32, device=DEV).repeat(M // 1000, 1)
    scale = torch.rand(M, K // 128, device=DEV) * 1e-3
    rows = torch.tensor([0, 1, 35001, 65535, 65537, 69999], device=DEV)
    w = GroupRows(q, scale, None, K, 4, 128)
    part = GroupRows(q[rows].contiguous(), scale[rows].contiguous(), None, K, 4, 128)
    for T in (1, 6, 70):
        x = torch.randn(T, K, device=DEV).to(torch.bfloat16)
        y, z = samd.group_matmul(x, w)[:, rows].double(), samd.group_matmul(x, part).double()
        assert (y - z).norm() <= 2.0 ** -8 * z.norm()
    # the gradient reads them too: only the chosen rows have a gradient
    dy = torch.zeros(2, M, device=DEV, dtype=torch.bfloat16)
    dy[:, rows] = torch.randn(2, len(rows), device=DEV).to(torch.bfloat16)
    a = samd.group_matmul_grad(dy, w).double()
    b = samd.group_matmul_grad(dy[:, rows].contiguous(), part).double()
    assert (a - b).norm() <= 2.0 ** -8 * b.norm()


def test_more_than_2_31_values_through_8_bits():
    rows, cols = 66000, 32776
    x = torch.empty(rows, cols, dtype=torch.float16, device=DEV)
    x.copy_(torch.randn(1000, cols, device=DEV).to(torch.float16).repeat(66, 1))
    r = samd.group_quantize(x, 8, True, 32)
    back = samd.group_dequantize(r, torch.float16)
    for i in (0, 32767, 65535, 65999):
        s = samd.group_quantize(x[i:i + 1].clone(), 8, True, 32)
        assert torch.equal(r.q[i:i + 1], s.q) and torch.equal(r.scale[i:i + 1], s.scale)
        assert torch.equal(back[i:i + 1], samd.group_dequantize(s, torch.float16))
