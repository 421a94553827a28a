"""The example that trains a 4-bit linear map from 8-bit batches and serves it by coded workers."""
import importlib.util
import os

import pytest

from tests.gpu_helpers import torch_mod

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx_linear.py")


@pytest.fixture(scope="module")
def example():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("mx_linear", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_from_saved_batches_reduces_the_error(example):
    losses, weights, d_batch = example.train(512, 200, 130, 20)
    # the map starts at zero: the first error is the targets' variance, 1; 4-bit weights stay some tenths off
    assert 0.8 < losses[0] < 1.2 and losses[-1] < 0.1 * losses[0]
    assert weights.shape == (130, 200) and bool(d_batch.float().isfinite().all())


@pytest.mark.parametrize("n,k,q,r,s", [(6, 4, 130, 200, 1), (16, 12, 500, 96, 3), (5, 3, 7, 33, 2)])
def test_coded_workers_recover_the_microscaled_product(example, lib, n, k, q, r, s):
    """Normwise 2e-2, the bound of the bf16 codes' products, against the product itself."""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(q)
    weights = lib.alloc_mx(q, r, lib.CODED_MX4)
    lib.coded_mx_quantize(torch.randn((q, r), generator=g, device="cuda"), weights)
    x = torch.randn((r, s), generator=g, device="cuda").to(torch.bfloat16)
    plain = torch.empty((q, s), device="cuda")
    lib.coded_mx_mm(weights, x, plain)
    for draw in range(4):
        out, survivors, info = example.serve(weights, x, n, k, seed=3, draw=draw)
        assert int(info.item()) == 0 and len(survivors) == k
        assert float((out - plain).abs().max() / plain.abs().max()) <= 2e-2
