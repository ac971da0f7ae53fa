"""Scores so large that one unit of theirs in 32 bits is many powers of two of a weight: no weight overflows, and outputs stay averages of values."""
import pytest
import torch

from attention_ref import BF16, F16, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("new,wide", [(1, 0), (1, 600), (90, 0), (90, 600)])
@pytest.mark.parametrize("size", [20, 23, 24, 25, 26, 27])
@pytest.mark.parametrize("run", [16, 48, 128, 300])
def test_rising_large_scores(ubp, dtype, new, wide, size, run):
    """Scores of 1.44 2^size (of a base 2) that rise by one step of the products' sums from one run of keys to the next."""
    n, D = 1400, 64
    b = Batch([new], [n], 2, 1, D, dtype, 16, wide=wide, seed=size)
    b.K[0].zero_()
    b.K[0][:, :, 0] = 2.0 ** 15                            # (f16 ends below 2^16)
    b.K[0][:, :, 1] = (torch.arange(n, device="cuda") // run).to(dtype)[:, None]
    b.V[0].copy_(1 + torch.rand(b.V[0].shape, generator=b.g, device="cuda"))
    b.write()
    q = torch.zeros(new, 2, D, dtype=dtype, device="cuda")
    q[:, :, 0] = 2.0 ** (size + 3 - 15)                        # sums of 2^(size + 3), over the root of 64
    q[:, 0, 1], q[:, 1, 1] = 2.0 ** max(size + 3 - 23, 3), 1.5 * 2.0 ** max(size + 3 - 23, 3)
    out = ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=new).double()
    # an average of the last run's values, whatever the weights: within their range, up to the rounding of the weights and the output
    low, high = b.V[0].double().amin((0, 1)), b.V[0].double().amax((0, 1))
    assert torch.isfinite(out).all()
    u = torch.finfo(dtype).eps
    assert ((out >= low * (1 - 2 * u)) & (out <= high * (1 + 2 * u))).all()
