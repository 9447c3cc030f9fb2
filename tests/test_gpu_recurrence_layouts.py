"""The recurrence on every layout of its work: one block a chain over several tiles, clusters, published maps with rows of 32
words and narrower ones, each with rows that come by tensor copies, by words, and straight from memory."""
import pytest

import test_gpu_recurrence as base

pytestmark = pytest.mark.gpu
mf = base.mf

# On 152 SMs, forward and backward.
SHAPES = [
    (160, 700, 128), (330, 300, 64), (170, 400, 100), (330, 300, 33),  # one block a chain, 3 to 6 tiles
    (40, 1500, 128), (40, 1500, 100), (40, 1500, 65),                  # clusters of 2, 6 rounds
    (20, 3000, 128), (20, 3000, 100), (20, 3000, 99),                  # clusters of 4
]
LONG = [
    (1, 40000, 64), (1, 30000, 40), (2, 30000, 33), (1, 20000, 7),     # published maps; rows narrowed to 8 words
    (1, 20000, 512),                                                   # published maps, rows by tensor copies
]


@pytest.mark.parametrize("dtype,marks", [("f32", "none"), ("f32", "mixed"), ("bf16", "none"), ("bf16", "mixed"), ("f16", "mixed")])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(mf, shape, dtype, marks):
    base._check(mf, shape, dtype, marks, seed=sum(shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LONG)
def test_few_long_chains(mf, shape, dtype):
    base._check(mf, shape, dtype, "mixed", seed=sum(shape))
