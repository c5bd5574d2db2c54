"""The 4-bit products at the end of the range that include/kvpipe.h states."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
from test_gpu_w4 import _linear, _normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("M", [1, 5, 33])
def test_largest_inputs(group, M):
    """Inputs of 2^118 throughout, of one sign (the codes' offset adds up to 1.5 times their sum): finite and right."""
    rng = np.random.default_rng(10)
    N, K = 40, 640
    codes, s = lr.w4_codes(lr.bf16(_normal(rng, N, K) * np.float32(2.0**-90)), group)
    buf = torch.from_numpy(lr.w4_pack(codes, s)).cuda()
    x = np.full((M, K), 2.0**118, np.float32)
    x[-1] *= lr.bf16(rng.uniform(0.5, 1, K).astype(np.float32))
    y = x.astype(np.float64) @ lr.w4_weights(codes, s, group).T
    got = _linear(x, buf, N, group)
    assert (np.abs(got - y) <= lr.linear_bound(x.astype(np.float64), y, s, group)).all()
