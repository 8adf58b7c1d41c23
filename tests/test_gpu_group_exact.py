"""Group-scaled rows on the GPU: what a result owes to the formula alone, against 64 bits.  The bounds count a weight as
its value |s (q - z)|, not as its fields, so that a weight equal to its zero point may not show in a result at all."""
import numpy as np
import pytest
import torch

import paper_1809_10572_amd as samd
from paper_1809_10572_amd import GroupRows
import group_reference as ref

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
