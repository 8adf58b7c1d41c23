"""What the GPU tests of 24-bit products take as their border, on the CPU: operands cut to 16 bits are beyond it, sums in
32-bit floats are not."""
import numpy as np
import pytest

BORDER = 2.0 ** -18


def cut(x, bits):
    """float32 values with all but their upper significant bits cleared."""
    return (x.view(np.uint32) & np.uint32(0xffffffff << (24 - bits) & 0xffffffff)).view(np.float32)


@pytest.mark.parametrize("K", [128, 700, 4400])
def test_border_of_24_bits(K):
    rng = np.random.default_rng(K)
    x = rng.standard_normal((40, K)).astype(np.float32)
    w = (rng.integers(-8, 8, (50, K)) * (rng.random((50, 1)) + 0.5)).astype(np.float32)
    want = x.astype(np.float64) @ w.astype(np.float64).T
    lost = cut(x, 16).astype(np.float64) @ w.astype(np.float64).T
    assert np.linalg.norm(lost - want) > 2 * BORDER * np.linalg.norm(want)
    # one product after another, each of three pieces, in one 32-bit sum: the most roundings there can be, each by
    # 2^-23 / sqrt 12 of the sum on average at most, 3 K of them of sums whose squares average K / 2: in all
    # 0.58 2^-24 sqrt(3 K / 2) of the result, 47 of the border's 64 units for K = 4400
    total = np.zeros(want.shape, dtype=np.float32)
    pieces, rest = [], x
    for _ in range(3):
        pieces.append(cut(rest, 8))
        rest = rest - pieces[-1]
    assert not rest.any()
    for k in range(K):
        for p in pieces:
            total += p[:, k, None] * w[None, :, k]
    assert np.linalg.norm(total - want) < BORDER * np.linalg.norm(want)
