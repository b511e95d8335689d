"""What the attention's weights hold to.

u = 2^-24.  Scores here are one product q k and its factors: off by 2 u of
themselves (log2 e, and one product).  2^x by the hardware is within 2^-22; a weight
in BF16 words is exact, in FP16 words within 2^-22.  A matrix instruction's sums may
be cut off instead of rounded: 2 u of the largest term each."""
import numpy as np
import pytest
import torch

from test_gpu_kv import BF16, F16, U, close, f64, half_eps, smallest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_weights_have_the_bits_of_fp32(pmpe, dtype):
    """Three positions whose values cancel the first two words of a weight: keys
    0, x, 0 and values -c1, 1, -c2 with c1 + c2 = e^x to two words of the type."""
    B, D = 96, 16
    x = (-torch.linspace(0.02, 0.68, B)).to(dtype)
    w = torch.exp(x.double())
    c1 = w.to(dtype)
    c2 = (w - c1.double()).to(dtype)
    c = pmpe.KvCache.empty(B, 16, 1, D, dtype)
    c.k[:, 0, 1, 0] = x.cuda()
    c.v[:, 0, 0] = -c1.cuda()[:, None]
    c.v[:, 0, 1] = 1.0
    c.v[:, 0, 2] = -c2.cuda()[:, None]
    q = torch.zeros((B, 1, D), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    a = c.attend(q, table, torch.full((B,), 3, dtype=torch.int32, device="cuda"), scale=1.0)
    w, x, rest = w.numpy(), np.abs(f64(x)), (w - c1.double() - c2.double()).numpy()
    want = rest / (2 + w)
    # the score's and the power's errors; three instructions' sums of terms up to 1, the four warps', the quotient's
    bound = (w * (2 * U * x + 2.0 ** -22) + (0 if dtype == BF16 else 2.0 ** -22) + 2 * 3 * U + 6 * U * np.abs(rest)) / (2 + w)
    close(f64(a.out[:, 0]), want[:, None], (bound + half_eps(dtype) * (np.abs(want) + bound) + smallest(dtype))[:, None])
