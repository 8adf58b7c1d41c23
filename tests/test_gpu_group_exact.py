"""Group-scaled rows on the GPU: what a result owes to the formula alone, against 64 bits.  The bounds count a weight as
its value |s (q - z)|, not as its fields, so that a weight equal to its zero point may not show in a result at all."""
import math

import pytest
import torch

import paper_1809_10572_amd as samd
from paper_1809_10572_amd import GroupRows

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"


def weights(gen, rows, cols, group, signed):
    """Random 4-bit rows: (GroupRows, 64-bit values)."""
    q = torch.randint(0, 16, (rows, cols), generator=gen, device=DEV)
    return from_fields(gen, q, group, None if signed else torch.randint(
        0, 16, (rows, -(-cols // group)), generator=gen, device=DEV).to(torch.uint8))


def from_fields(gen, q, group, zero, scale=None):
    """Rows of the given fields 0..15 (signed where zero is None, in two's complement)."""
    rows, cols = q.shape
    wide = torch.nn.functional.pad(q, (0, -cols % 8))
    words = (wide.view(rows, -1, 8) << torch.arange(0, 32, 4, device=DEV)).sum(2)
    words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
    groups = -(-cols // group)
    if scale is None:
        scale = (torch.rand(rows, groups, generator=gen, device=DEV) + 0.5) / (4 * cols ** 0.5)
    at = torch.arange(cols, device=DEV) // group
    whole = torch.where(q >= 8, q - 16, q) if zero is None else q - zero.long()[:, at]
    return GroupRows(words, scale, zero, cols, 4, group), scale.double()[:, at] * whole


def matrix(gen, rows, cols, typ):
    t = torch.randn(rows, cols, generator=gen, device=DEV).to(TYPES[typ])
    return t, t.double()


# tokens for every kernel of the products and of the gradient
TOKENS = [1, 2, 3, 16, 20, 70, 300]


# ---- zero points at any address -------------------------------------------------------------------

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", TOKENS)
def test_zero_points_at_any_byte(T, group):
    """Odd numbers of rows and groups, zero points that start 1 to 3 bytes behind a word and end anywhere: the results
    are those of zero points on a word."""
    gen = torch.Generator(device=DEV).manual_seed(T + group)
    M, K = 37, 3 * group - 5
    wg, wu = weights(gen, M, K, group, False)[0], weights(gen, M, K, group, False)[0]
    for typ in TYPES:
        x, dy = matrix(gen, T, K, typ)[0], matrix(gen, T, M, typ)[0]
        y, h, dx = samd.group_matmul(x, wg), samd.group_gated(x, wg, wu), samd.group_matmul_grad(dy, wg, dy, wu)
        for off in (1, 2, 3):
            def moved(w):
                z = torch.full((w.zero.numel() + 8,), 255, dtype=torch.uint8, device=DEV)[off:off + w.zero.numel()]
                return w._replace(zero=z.copy_(w.zero.flatten()).view(w.zero.shape))
            vg, vu = moved(wg), moved(wu)
            assert vg.zero.data_ptr() % 4 == off
            assert torch.equal(samd.group_matmul(x, vg), y), (typ, off)
            assert torch.equal(samd.group_gated(x, vg, vu), h), (typ, off)
            assert torch.equal(samd.group_matmul_grad(dy, vg, dy, vu), dx), (typ, off)


# ---- weights equal to their zero points -----------------------------------------------------------

def rounding(typ, want):
    """The rounding of 64-bit results to a type: half a step of their value, and, below the type's smallest normal number
    m, where steps no longer shrink, half of m eps: for f16 2^-14 2^-10 / 2 = 2^-25."""
    t = torch.finfo(TYPES[typ])
    return torch.clamp(want.abs(), min=t.smallest_normal) * (t.eps / 2)


def near_zero_points(gen, rows, cols, group, zero, ones):
    """Rows whose fields all equal their zero point, but for `ones` of each row, which lie one step above (below, where the
    zero point is 15)."""
    groups = -(-cols // group)
    if zero == "any":
        z = torch.randint(0, 16, (rows, groups), generator=gen, device=DEV)
    else:
        z = torch.full((rows, groups), 8 if zero is None else zero, device=DEV)
    q = z.repeat_interleave(group, 1)[:, :cols].clone()
    if ones:
        at = torch.randint(0, cols, (rows, ones), generator=gen, device=DEV)
        q.scatter_(1, at, q.gather(1, at) + torch.where(q.gather(1, at) == 15, -1, 1))
    if zero is None:
        q = q ^ 8   # two's complement of the field less 8
    return from_fields(gen, q, group, None if zero is None else z.to(torch.uint8))


def product_is_the_formulas(typ, T, K, M=70):
    """Nothing from weights that are nothing, and a bound that counts the others alone: at most K/32 + 64 additions and
    roundings of 2^-24 each of the sum of their magnitudes, and the result's rounding."""
    gen = torch.Generator(device=DEV).manual_seed(T + K)
    # of one sign, over twelve powers of two: sums whose bits do not all fit, whatever the type
    x = torch.exp2(12 * torch.rand(T, K, generator=gen, device=DEV) - 10).to(TYPES[typ])
    for group in (32, 64, 128):
        for zero in (None, 0, 3, 15, "any"):
            w, _ = near_zero_points(gen, M, K, group, zero, 0)
            assert not samd.group_matmul(x, w).any(), (group, zero)
            assert not samd.group_gated(x, w, w).any(), (group, zero)
            w, values = near_zero_points(gen, M, K, group, zero, 3)
            want = x.double() @ values.t()
            bound = rounding(typ, want) + (K / 32 + 64) * 2.0 ** -24 * (x.double() @ values.abs().t())
            off = ((samd.group_matmul(x, w).double() - want).abs() - bound).max().item()
            assert off <= 0, (group, zero, off)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [256, 2051, 4100])
@pytest.mark.parametrize("T", [1, 2])
def test_products_of_one_and_two_tokens(typ, T, K):
    product_is_the_formulas(typ, T, K)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [256, 2051, 4100])
@pytest.mark.parametrize("T", [3, 16, 20, 70, 300])
def test_products_of_more_tokens(typ, T, K):
    product_is_the_formulas(typ, T, K)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_wide_products_of_few_tokens(typ):
    """So many rows that a workgroup takes 32 of them."""
    product_is_the_formulas(typ, 5, 260, 8200)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 5, 20, 600])
def test_zero_points_beyond_the_fields(typ, T):
    """Zero points are bytes: differences down to -255 are whole numbers too."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    M, K = 300, 421
    x, xv = matrix(gen, T, K, typ)
    dy, dyv = matrix(gen, T, M, typ)
    for group in (32, 64, 128):
        q = torch.randint(0, 16, (M, K), generator=gen, device=DEV)
        zero = torch.randint(0, 256, (M, -(-K // group)), generator=gen, device=DEV).to(torch.uint8)
        zero[:, 0] = torch.arange(M, device=DEV) % 256
        w, values = from_fields(gen, q, group, zero)
        want, size = xv @ values.t(), xv.abs() @ values.abs().t()
        bound = rounding(typ, want) + (K / 32 + 64) * 2.0 ** -24 * size
        off = ((samd.group_matmul(x, w).double() - want).abs() - bound).max().item()
        assert off <= 0, (group, off)
        want, size = dyv @ values, dyv.abs() @ values.abs()
        bound = rounding(typ, want) + (LOST[typ] + (M / 32 + 64) * 2.0 ** -24) * size
        off = ((samd.group_matmul_grad(dy, w).double() - want).abs() - bound).max().item()
        assert off <= 0, ("dx", group, off)


# What a product dy w may lose on its way into a gradient, as a part of it.  bf16: the weight rounded to a bf16, 2^-8.
# f16: both cut to 8 bits, what is cut off below 2^-7 of each (of dy's 11 bits, at most 7/8 of that); the weight's cut-off
# part is rounded to 8 bits, 2^-8 of at most 2^-8 where it is largest, 2^-16; the product of the cut-off parts is left out,
# 7/8 2^-14; together 9/8 2^-14.  f32: pieces below 1, 2^-7 and 2^-15 of each, exact; left out are the second by the third,
# twice, and the third by the third: 2 2^-22 + 2^-30; and the weight's own product with its scale, 2^-24.
LOST = {"f32": 2.0 ** -21 + 2.0 ** -23, "f16": 1.125 * 2.0 ** -14 + 2.0 ** -23, "bf16": 2.0 ** -8 + 2.0 ** -23}


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(3, 300, 70), (40, 2051, 70), (600, 300, 260), (2040, 200, 4090)])
def test_gradients_are_the_formulas(typ, size):
    """Few and many tokens, for every tile of the gradient: nothing from weights that are nothing, and the bound of
    products with what the products themselves may lose."""
    T, M, K = size
    gen = torch.Generator(device=DEV).manual_seed(T + K)
    dy = torch.exp2(12 * torch.rand(T, M, generator=gen, device=DEV) - 10).to(TYPES[typ])
    for group in (32, 64, 128):
        for zero in (None, 3, 15, "any"):
            w, _ = near_zero_points(gen, M, K, group, zero, 0)
            assert not samd.group_matmul_grad(dy, w).any(), (group, zero)
            assert not samd.group_matmul_grad(dy, w, dy, w).any(), (group, zero)
            w, values = near_zero_points(gen, M, K, group, zero, 3)
            want, size = dy.double() @ values, dy.double() @ values.abs()
            bound = rounding(typ, want) + (LOST[typ] + (M / 32 + 64) * 2.0 ** -24) * size
            off = ((samd.group_matmul_grad(dy, w).double() - want).abs() - bound).max().item()
            assert off <= 0, (group, zero, off)


# ---- the activations' tails -----------------------------------------------------------------------

def activation_of(g, act):
    """act(g), act'(g) and the terms that the latter is the sum of, in 64 bits and without cancellation."""
    if act == "silu":
        e = torch.exp(-g.abs())
        p, q = torch.where(g < 0, e, 1.0) / (1 + e), torch.where(g < 0, 1.0, e) / (1 + e)   # p(g) and p(-g) = 1 - p(g)
        return g * p, (p, p * g * q)
    p = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))
    return g * p, (p, g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi))


def activation_bounds(g, act):
    """What 32-bit arithmetic may lose of act(g) and of act'(g).  gelu: the argument g / sqrt 2 is off by 1.5 2^-24 of
    itself, its constant and its product, which erfc turns into g^2 + 1 times as much at most; erfc itself by 16 last places, 32
    units of 2^-24; two products.  Its density: g^2 / 2 off by 2^-24 of itself, which the exponential turns into as much,
    the exponential by 2 last places, three products.  silu: the exponential, a sum, a quotient and a product; the slope's
    p (1 + g (1 - p)) the same for terms of p and p g; the exponential's steps of 2^-149 below 2^-126."""
    value, (p, rest) = activation_of(g, act)
    if act == "silu":
        off = 8 * 2.0 ** -24 * p + 2.0 ** -149
        return value, g.abs() * off, p + rest, (1 + g.abs()) * off
    rel, rel_rest = 1.5 * (g * g + 1) + 36, 0.5 * g * g + 10
    unit = 2.0 ** -24
    return value, value.abs() * rel * unit, p + rest, (p.abs() * rel + rest.abs() * rel_rest + (p + rest).abs()) * unit


def one_hot_rows(gen, at, M):
    """M rows of 32 weights that are 0 but for a 1 at k = at, of scale 1."""
    q = torch.zeros(M, 32, dtype=torch.long, device=DEV)
    q[:, at] = 1
    return from_fields(gen, q, 32, None, torch.ones(M, 1, device=DEV))[0]


def tail_of_gated(typ, act, g):
    """h = act(g) u for given g and u = 512, tokens enough for each kernel; and the stored form's h."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    want, off, _, _ = activation_bounds(g, act)
    want, off = 512 * want, 512 * off
    bound = rounding(typ, want) + off + 2.0 ** -24 * want.abs() + 512 * 2.0 ** -149
    for M in (1, 5):
        wg, wu = one_hot_rows(gen, 0, M), one_hot_rows(gen, 1, M)
        for T in (1, 2, 5, 20, 600):
            for i in range(0, len(g), T):
                x = torch.zeros(T, 32, dtype=TYPES[typ], device=DEV)
                n = min(T, len(g) - i)
                x[:n, 0], x[:, 1] = g[i:i + n].to(TYPES[typ]), 512
                for h in (samd.group_gated(x, wg, wu, act), samd.group_gated_save(x, wg, wu, act)[0]):
                    err = (h[:n].double() - want[i:i + n, None]).abs() - bound[i:i + n, None]
                    assert err.max() <= 0, (M, T, g[i + err.max(1)[0].argmax()].item())


def tail_of_gated_grad(typ, act, g, step):
    """dg and du for g = -step q in stored form, u = 512, dh = 1."""
    value, off, slope, off_slope = activation_bounds(g, act)
    n = len(g)
    q8 = torch.zeros(n, 4, dtype=torch.int8, device=DEV)
    q8[:, 0] = (g / step).round().to(torch.int8)
    u8 = torch.zeros_like(q8)
    u8[:, 0] = 64
    g8 = GroupRows(q8.view(torch.int32), torch.full((n, 1), step, device=DEV), None, 1, 8, 32)
    u8 = GroupRows(u8.view(torch.int32), torch.full((n, 1), 8.0, device=DEV), None, 1, 8, 32)
    dg, du = samd.group_gated_grad(torch.ones(n, 1, dtype=TYPES[typ], device=DEV), g8, u8, act)
    err = (dg[:, 0].double() - 512 * slope).abs() - (rounding(typ, 512 * slope) + 512 * off_slope + 2.0 ** -23 * 512 * slope.abs())
    assert err.max() <= 0, ("dg", g[err.argmax()].item())
    err = (du[:, 0].double() - value).abs() - (rounding(typ, value) + off + 2.0 ** -24 * value.abs())
    assert err.max() <= 0, ("du", g[err.argmax()].item())


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_gelu_keeps_its_tail(typ):
    g = -torch.arange(0, 97, device=DEV).double() / 8   # 0 .. -12, exact in every type
    tail_of_gated(typ, "gelu", g)
    tail_of_gated_grad(typ, "gelu", g, 0.125)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_silu_keeps_its_tail(typ):
    g = 4.0 - torch.arange(0, 105, device=DEV).double()   # 4 .. -100
    tail_of_gated(typ, "silu", g)
    tail_of_gated_grad(typ, "silu", g, 1.0)


# ---- f32 keeps 24 bits ----------------------------------------------------------------------------

def relative(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


# As test_group_precision shows for the CPU, operands cut to 16 bits put a whole result off by some 200 units of 2^-24 of its
# norm; sums of K products in 32-bit floats, if each of the K (and three times as many pieces) were rounded alone, by
# 0.58 sqrt(3 K / 2) at most on average: 47 for K = 4400.  The border lies between.
KEPT = 2.0 ** -18

# tokens, rows, columns, each tile of the products (rows of the result, summed columns) and of the gradient (summed rows)
PRECISE = [(1, 500, 4400), (2, 300, 2051), (3, 70, 2304), (16, 500, 1024), (20, 300, 4100), (70, 1013, 2051), (128, 128, 128),
           (300, 1100, 700), (510, 2000, 1100), (1000, 2100, 1096), (2040, 4090, 576), (2048, 4096, 1330)]


@pytest.mark.parametrize("size", PRECISE)
def test_f32_keeps_24_bits(size):
    T, M, K = size
    gen = torch.Generator(device=DEV).manual_seed(T + M)
    for group in (32, 64, 128):
        for signed in (True, False):
            w, values = weights(gen, M, K, group, signed)
            x, xv = matrix(gen, T, K, "f32")
            want = xv @ values.t()
            assert relative(samd.group_matmul(x, w), want) <= KEPT, (group, signed)
            v, other = weights(gen, M, K, group, signed)
            u = xv @ other.t()
            h = want / (1 + torch.exp(-want)) * u
            # three results of the kind, each off by as much at most, the activation's slope at most 1.1
            assert relative(samd.group_gated(x, w, v), h) <= 3.3 * KEPT, (group, signed)
            assert relative(samd.group_gated_save(x, w, v)[0], h) <= 3.3 * KEPT, (group, signed)
            # sums over K rows, as deep as the products' are
            w, values = weights(gen, K, M, group, signed)
            v, other = weights(gen, K, M, group, signed)
            dy, dyv = matrix(gen, T, K, "f32")
            want = dyv @ values
            assert relative(samd.group_matmul_grad(dy, w), want) <= KEPT, (group, signed)
            assert relative(samd.group_matmul_grad(dy, w, x, v), want + xv @ other) <= KEPT, (group, signed)


# ---- projections that cannot be stored ------------------------------------------------------------

@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [4, 70, 600])
def test_stored_rows_of_nothing_and_of_no_number(typ, T):
    """A token of zeros is stored as zeros of scale 0, one with an infinity or a NaN as words of 0 and scales of NaN; the
    other tokens as without them."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    for M, K, group in ((45, 90, 32), (700, 256, 128)):
        wg, wu = weights(gen, M, K, group, False)[0], weights(gen, M, K, group, False)[0]
        x, _ = matrix(gen, T, K, typ)
        x[0] = 0
        h, g, u = samd.group_gated_save(x, wg, wu)
        assert not h[0].any()
        for r in (g, u):
            assert not r.q[0].any() and not r.scale[0].any() and (r.scale[1:] > 0).all()
        bad = {1: float("inf"), T // 2: float("nan"), T - 1: float("-inf")}
        for t, v in bad.items():
            x[t, t % K] = v
        h2, g2, u2 = samd.group_gated_save(x, wg, wu)
        rest = torch.tensor([t not in bad for t in range(T)], device=DEV)
        assert torch.equal(h2[rest], h[rest]) and not torch.isfinite(h2[~rest]).any()
        for r, r2 in ((g, g2), (u, u2)):
            assert torch.equal(r2.q[rest], r.q[rest]) and torch.equal(r2.scale[rest], r.scale[rest])
            assert not r2.q[~rest].any() and torch.isnan(r2.scale[~rest]).all()
            assert torch.isnan(samd.group_dequantize(r2)[~rest]).all()
        dg, du = samd.group_gated_grad(torch.ones_like(h2), g2, u2)
        assert torch.isnan(dg[~rest]).all() and torch.isnan(du[~rest]).all()
        assert torch.isfinite(dg[rest]).all() and torch.isfinite(du[rest]).all()
