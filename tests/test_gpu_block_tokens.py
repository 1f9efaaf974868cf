"""The residual block for one to three tokens of each entry, as generation calls it: many entries, any number of channels."""
import pytest

from test_gpu_block import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", [(32, 768, 1), (1, 768, 1), (7, 5, 1), (3, 40, 1), (5, 300, 1), (2, 1030, 1), (3, 2048, 1), (2, 2100, 1), (700, 20, 1), (9, 130, 2), (6, 600, 3)],
                         ids=str)
def test_few_tokens(B, C, T, dtype):
    check(B, C, T, dtype, seed=B + C)
    check(B, C, T, dtype, "sigmoid", post=False, p=0.2, seed=B + C + 1, site=1)
    check(B, C, T, dtype, "none", pre=False, seed=B + C + 2)
