"""The operators beside the sparse product on the GPU: values at the borders of what the header defines, in every path."""
import numpy as np
import pytest
import torch

import paper_2506_15174_amd as spmm
from layers_reference import HALF_STEP, SMALLEST, TYPES, act64, as64, codes_of, placed, summed, weights

pytestmark = pytest.mark.gpu

FLOATS = ("float32", "float16", "bfloat16")
# features, tokens, order in memory: one wave a token, one workgroup of 256 or 1024, long rows; rows of features in one launch and in two
ROWS_PATHS = [(40, 6, "tokens"), (2000, 3, "tokens"), (4100, 3, "tokens"), (8000, 600, "tokens"), (16000, 3, "tokens"), (33000, 3, "tokens"), (70000, 2, "tokens"),
              (40, 6, "features"), (1024, 128, "features"), (4096, 6, "features"), (5000, 6, "features"), (3000, 270, "features")]


@pytest.fixture(autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spmm.load()


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("K,N,order", ROWS_PATHS)
def test_codes_of_a_token_of_zeros_without_eps(type, K, N, order):
    """P is 0: codes and scale are 0 whatever eps is; so they are where the weights make it 0."""
    x = placed(np.random.default_rng(K).standard_normal((K, N)), type, order)
    x[:, 0] = 0
    w = torch.ones(K, device="cuda")
    for eps in (0.0, 1e-6):
        y = spmm.norm(x, w, eps, dtype=torch.int8)
        assert y.scales[0] == 0 and (y.out[:, 0] == 0).all() and y.scales.isfinite().all() and (y.scales[1:] > 0).all()
        n = spmm.norm(x, torch.zeros_like(w), eps, dtype=torch.int8)
        assert (n.scales == 0).all() and (n.out == 0).all()
    g = spmm.gate(x, x, dtype=torch.int8)
    assert g.scales[0] == 0 and (g.out[:, 0] == 0).all() and (g.scales[1:] > 0).all()
