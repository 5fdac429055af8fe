"""GPU parity of the Newton-Schulz orthogonalisation for entries far below the largest, element by element: X is kept with 22 bits from step
to step, and nothing of it is finer than 2^-46."""
import pytest
import torch

from tests.test_gpu_orthogonalise import formula, matrix, orthogonalise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(60, 200), (60, 1400), (130, 264), (300, 70), (1030, 1100), (96, 4100)])
@pytest.mark.parametrize("size", [1e-4, 1e-6, 1e-7, 1e-8, 1e-9, 1e-10])
def test_small_singular_values_beside_a_large_one(rows, cols, size):
    """One large entry and small ones, each the only one of its row and column: the small ones are its singular values, and each
    goes through the five steps by itself.  A step multiplies by a = 3.4445, so of the errors that the steps leave in units of
    2^-46 the first counts most, 1 / (1 - 1 / a) = 1.41 of it in all; the store in bf16 takes at most 2^-8, and sums, products and 22
    bits together less than 1e-4."""
    print(f"[case] orthogonalise {rows} x {cols}, entries of {size}", flush=True)
    u = torch.zeros(rows, cols)
    n = min(rows, cols)
    u[torch.arange(n), torch.arange(n)] = size * (1.0 + matrix(1, n).abs()[0])
    u[0, 0] = 1.0
    got, ref = orthogonalise([u], eps=0.0)[0].cpu().double(), formula(u, eps=0.0)
    some = ref != 0
    assert (got[~some] == 0).all()
    over = (got - ref).abs()[some] / ref.abs()[some]
    assert over[1:].max() <= 2.0 ** -8 + 1.5 * 2.0 ** -46 / size + 1e-4, float(over[1:].max())
