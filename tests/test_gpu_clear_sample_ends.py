"""Rows of logits at both ends of 32 bits: two of them may be further apart than the largest number, which at temperatures near it is a distance like any other.  Against the definition in
64 bits, with every filter and every form of the kernels: short rows, long ones, rows over several workgroups, bounds among candidates and in the row itself."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_clear_sample import TYPES, check, ctx  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(60, 2500), (24, 40000), (300, 17000), (1030, 17000), (8, 131072)])
def test_logits_at_both_ends(ctx, kind, rows, vocab):  # noqa: F811
    rng = np.random.default_rng(rows + vocab)
    x = torch.from_numpy(rng.uniform(-3.3e38, 3.3e38, (rows, vocab)).astype(np.float32)).to(TYPES[kind])
    check(ctx, x, rng.random(rows), rng.choice([1e37, 5e37, 1e38, 3.4e38], rows), rng.choice([0, 0, 40, vocab // 3, vocab - 1], rows), rng.choice([1, 0.5, 0.9, 0.99], rows), rng.choice([0, 0, 0.01, 0.3], rows))


def test_two_logits(ctx):  # noqa: F811
    """The lower one weighs exp(-2) of the higher: whichever filter leaves both, both are drawn."""
    x = torch.tensor([[3e38, -3e38]]).repeat(8, 1)
    u = [0.5, 0.88, 0.89, 0.99] * 2
    for k, p, m in ((0, 1, 0), (0, 0.95, 0), (2, 0.95, 0), (0, 1, 0.1), (0, 0.95, 0.1), (3, 1, 0)):
        check(ctx, x, u, 3e38, k, p, m)
    wide = torch.full((8, 5000), -3e38)
    wide[:, 4321] = 3e38
    for k in (1, 2, 4999, 0):
        check(ctx, wide, u, 3e38, k, 0.95, 0)
