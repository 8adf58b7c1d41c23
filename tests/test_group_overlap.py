"""Results that share memory with operands, without a GPU: refused, and rows that only lie between each other's are not."""
import random

import pytest
import torch

import paper_1809_10572_amd as samd
from test_group_checks import fake, rows   # noqa: F401 (a fixture)


def bytes_of(base, t):
    """The bytes of a two-dimensional tensor, counted from the buffer's start."""
    first = t.data_ptr() - base
    return {first + i * t.stride(0) * t.element_size() + j for i in range(t.shape[0]) for j in range(t.shape[1] * t.element_size())}


def test_whether_two_tensors_meet():
    rng, buf = random.Random(3), torch.zeros(400)
    base, both = buf.data_ptr(), {True: 0, False: 0}

    def view():
        cols = rng.randint(1, 9)
        step = cols + rng.choice([0, 0, 1, 5, 12])
        return torch.as_strided(buf, (rng.randint(1, 9), cols), (step, 1), rng.randint(0, 150))

    for i in range(4000):
        a, b = view(), view()
        if i % 2:   # the same step, as two halves of the columns of one buffer have
            b = torch.as_strided(buf, b.shape, (max(a.stride(0), b.shape[1]), 1), b.storage_offset())
        meet = bool(bytes_of(base, a) & bytes_of(base, b))
        both[meet] += 1
        assert samd._meet(a, b) == meet and samd._meet(b, a) == meet, (a.shape, a.stride(), b.shape, b.stride())
    assert min(both.values()) > 800
    assert not samd._meet(torch.zeros(0, 4), buf) and not samd._meet(buf[:0], buf)


def test_overlapping_results_are_refused(fake):
    rec, _ = fake
    x, w = torch.zeros(4, 64), rows(64, 64)
    g, u = rows(4, 64, 8), rows(4, 64, 8)
    buf = torch.zeros(4, 128)
    dy, other = torch.zeros(4, 64), torch.zeros(4, 64)
    words = torch.zeros(64, 8, dtype=torch.int32)
    bad = [
        lambda: samd.group_matmul(x, w, out=x),
        lambda: samd.group_matmul(buf[:, :64], w, out=buf[:, 60:124]),
        lambda: samd.group_matmul(x[:2], w, out=x[1:3]),
        lambda: samd.group_matmul(x, w._replace(scale=buf.view(-1)[:128].view(64, 2)), out=buf[:, 64:]),
        lambda: samd.group_matmul_grad(dy, w, out=dy),
        lambda: samd.group_matmul_grad(dy, w, other, w, out=other),
        lambda: samd.group_gated(x, w, w, out=x),
        lambda: samd.group_gated_save(x, w, w, out=x),
        lambda: samd.group_gated_grad(dy, g, u, out=(dy, other)),
        lambda: samd.group_gated_grad(dy, g, u, out=(other, other)),
        lambda: samd.group_gated_grad(dy, g, u, out=(other, dy)),
        lambda: samd.group_dequantize(rows(8, 64)._replace(q=words[:8]), out=words.view(torch.float32).view(8, 64)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert not rec.calls, i
    # neighbours in one buffer are no overlap
    samd.group_matmul(buf[:, :64], w, out=buf[:, 64:])
    samd.group_matmul(x[:2], w, out=x[2:])
    samd.group_gated_grad(dy, g, u, out=(buf[:, :64], buf[:, 64:]))
    samd.group_matmul_grad(dy, w, dy, w, out=other)   # inputs may be the same tensor
    assert len(rec.calls) == 4
