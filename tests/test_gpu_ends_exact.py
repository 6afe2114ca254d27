"""GPU embedding, dropout and class loss where results can be said exactly or nearly so: the order of an embedding's sums,
products of every number of steps, losses of rows that are sure of their label."""

import pytest

from tests.test_gpu_ends import loss_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
def test_loss_products_of_every_number_of_steps(gt, dtype, steps):
    # the sum over the features, over the classes and over the rows in one to five steps of 128 bytes: the first step
    # stands alone or in a pair, and its operands have landed in either case
    k = steps * (64 if dtype == "bf16" else 32)
    for n, V, D in ((33, 40, k), (300, 300, k), (1100, 3000, k), (40, k, 96), (k, 70, 64), (250, k, 700)):
        loss_case(gt, n, V, D, dtype, labelled=1.0 if n <= 256 else 0.7, seed=n + V + D)
