"""What a plan of the token-major product keeps, and on which streams it may be built and used."""
import pytest
import torch

from linear_ref import make_weight

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def resident_bytes():
    with open("/proc/self/statm") as f:
        return int(f.read().split()[1]) * 4096


def test_no_host_copy_of_the_image_stays(ubp):
    """An image of 160 MB: once it is on the device nothing on the host reads it again."""
    W, mask = make_weight(8192, 8192, 4, 90, 3)
    blob = ubp.ubp_pack(W, mask, 4)
    del W, mask
    small, sm = make_weight(64, 64, 4, 50, 3)
    first = ubp.LinearPlan(ubp.ubp_pack(small, sm, 4), BF16)      # (what the device and the allocator set up once)
    torch.cuda.synchronize()
    before = resident_bytes()
    plan = ubp.LinearPlan(blob, BF16)
    torch.cuda.synchronize()
    grown = resident_bytes() - before
    assert plan.dev_bytes > 140 << 20 and grown < plan.dev_bytes // 2, grown
    assert first.dev_bytes < 1 << 20
