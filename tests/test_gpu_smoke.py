"""The smoke step runs what it says: every kernel of the token-major product."""
import pytest

pytestmark = pytest.mark.gpu


def test_smoke_reaches_every_kernel_of_the_product(monkeypatch, capsys):
    import __graft_entry__
    import paper_2407_19644_b200 as ubp
    taken, call = set(), ubp.ubp_linear
    monkeypatch.setattr(ubp, "ubp_linear", lambda plan, x, **k: taken.add(plan.choice(x.shape[0])) or call(plan, x, **k))
    __graft_entry__.smoke()
    assert {k for k, _, _ in taken} == {0, 1, 2} and any(k == 1 and split > 1 for k, _, split in taken), taken
    assert "smoke ok" in capsys.readouterr().out
