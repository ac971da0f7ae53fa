"""Rows that see no key give 0, whatever the keys and values hold that other rows of the sequence see."""
import pytest
import torch

from attention_ref import BF16, F16, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("max_new,wide,Hq,pad", [(2, 0, 4, 0), (2, 600, 4, 0), (2, 600, 80, 0), (100, 0, 4, 0), (100, 600, 4, 0), (100, 0, 4, 1)])
def test_rows_before_the_sequence(ubp, dtype, value, max_new, wide, Hq, pad):
    """More new tokens than the sequence is long: those before position 0 see nothing, the last ones see infinities."""
    b = Batch([3, 2, 5], [2, 1, 0], Hq, 2, 64, dtype, 16, wide=wide)
    for v in b.V:
        v[:] = value
    b.write()
    q = b.queries()
    buf = torch.full((b.T, Hq, 64 + pad), -77.0, dtype=dtype, device="cuda")      # (pad: rows of the output off 16 bytes)
    out = ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=max_new, out=buf[:, :, :64])
    nothing = [0, 3, 5, 6, 7, 8, 9]
    assert (out[nothing] == 0).all()
    assert not torch.isfinite(out[[1, 2, 4]]).any()


@pytest.mark.parametrize("new", [[1] * 9, [30] + [1] * 8])
def test_rows_before_the_sequence_with_a_prefix(ubp, new):
    """The same where the shared prefix is read once: the last sequence has no tokens yet."""
    prefix = 58610
    b = Batch(new, [prefix + 50] * 8 + [0], 2, 1, 64, BF16, 16, prefix=prefix)
    b.V[0][7] = float("inf")
    for v in b.V[1:8]:
        v[7] = float("inf")
    b.write()
    out = ubp.ubp_prefix_attention(b.queries(), *b.args(), prefix, starts=b.starts, max_new=max(new))
    assert (out[b.first[8]] == 0).all() and torch.isinf(out[:b.first[8]]).all()
