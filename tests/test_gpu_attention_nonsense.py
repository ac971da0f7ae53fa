"""Numbers on the device that make no sense: no access out of range, and what comes after is right."""
import pytest
import torch

from attention_ref import BF16, Batch, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


@pytest.mark.parametrize("max_new", [None, 1])
def test_starts_whose_steps_pass_32_bits(ubp, max_new):
    """Every other sequence claims all rows, each with a million tokens before it: nothing is done."""
    T, B, page, width = 65536, 2400, 1 << 15, 32
    k, v = (torch.zeros(1, 1, page, 8, dtype=BF16, device="cuda") for _ in range(2))
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    lengths = torch.full((B,), page * width, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, T] * (B // 2) + [0], dtype=torch.int32, device="cuda")
    q, out = torch.zeros(T, 1, 8, dtype=BF16, device="cuda"), torch.full((T, 1, 8), 5.0, dtype=BF16, device="cuda")
    ubp.ubp_attention(q, k, v, table, lengths, starts=starts, max_new=max_new, out=out)
    ubp.attention_check()
    assert (out == 5.0).all()


def test_starts_that_do_not_ascend(ubp):
    """Rows that two sequences claim have the result for one of them; the others their own."""
    b = Batch([6, 5, 4], [60, 50, 40], 4, 2, 64, BF16, 16)
    q = b.queries()
    b.starts[1], b.starts[2] = 9, 4                            # rows 0 .. 8, none, 4 .. 14
    for max_new in (None, 1):
        out = ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=max_new)
        assert torch.isfinite(out).all()
    b = Batch([6, 5, 4], [60, 50, 40], 4, 2, 64, BF16, 16)
    q = b.queries()
    want, tol = b.exact(q)
    check(ubp.ubp_attention(q, *b.args(), starts=b.starts), want, tol, b.T)


@pytest.mark.parametrize("pad", [0, 3])
def test_a_sequence_that_has_outgrown_its_table(ubp, pad):
    """Its tokens keep their positions, those behind the table's end are not appended, and none takes an earlier one's place."""
    b = Batch([3, 2], [50, 20], 2, 1, 64, BF16, 16)            # (64 places each)
    b.len_t[0] = 66                                             # positions 63, 64, 65
    buf = torch.randn(5, 4 * 64 + pad, generator=b.g, device="cuda").to(BF16)
    qkv, rot = buf[:, :4 * 64], ubp.rotation_table(80, 64)
    b.table[0] = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    b.table[1, 0:2] = torch.tensor([4, 5], dtype=torch.int32)
    b.table[1, 2:] = -1
    b.k.zero_()
    q = ubp.ubp_rotate_append(qkv, 2, *b.args(), starts=b.starts, rotation=rot)
    changed = (b.k != 0).any(3)[:, 0]
    assert changed.nonzero().tolist() == [[3, 15], [5, 2], [5, 3]]
    wide = torch.cat([b.table, torch.full((2, 1), -1, dtype=torch.int32, device="cuda")], 1)
    assert torch.equal(ubp.ubp_rotate_append(qkv, 2, b.k, b.v, wide, b.len_t, starts=b.starts, rotation=rot), q)
    for max_new in (None, 1):
        out = ubp.ubp_attention(b.queries(), b.k, b.k, b.table, b.len_t, starts=b.starts, max_new=max_new)
        assert torch.isfinite(out).all()
