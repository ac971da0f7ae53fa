"""The operators of a pruned decoder layer together, as a serving program calls them: prompts, then answers from a captured graph."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kw", [
    dict(prompts=[1], tokens=4),
    dict(prompts=[300, 17, 129], tokens=5, window=40, sinks=3),
    dict(prompts=[2, 260], tokens=3, heads=6, kv_heads=1, size=80, width=384, page=8),
    dict(prompts=[513], tokens=2, heads=4, kv_heads=4, size=128, page=64)])
def test_layer_against_float64(kw):
    """bf16 activations and weights through four products, two norms and a softmax: each rounding at most 2^-8 of its value, about
    a dozen on the way, which add up like independent errors (12^(1/2) 2^-8 = 1.4 %), most of a row's size coming from the
    residual stream (unit variance beside sums of two parts of at most that)."""
    from examples.pruned_decoder_layer import run
    assert run(**kw) < 0.02


def test_example_runs():
    r = subprocess.run([sys.executable, os.path.join("examples", "pruned_decoder_layer.py")], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "pruned decoder layer ok" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


def test_prefix_in_a_layer():
    """Answers to one instruction: with the prefix told apart the layer's attention gives the same values to the rounding of the
    outputs (2^-8 of a value on either side, sums in another order)."""
    import paper_2407_19644_b200 as ubp
    g = torch.Generator(device="cuda").manual_seed(5)
    B, Hq, Hkv, D, P, prefix = 5, 8, 2, 64, 16, 96
    k, v = (torch.randn(64, Hkv, P, D, device="cuda", generator=g).bfloat16() for _ in range(2))
    table = torch.zeros(B, 10, dtype=torch.int32, device="cuda")
    table[:, :6] = torch.arange(6, device="cuda")
    table[:, 6:] = 6 + torch.arange(4 * B, device="cuda").view(B, 4)
    lengths = torch.tensor([97, 100, 112, 130, 160], dtype=torch.int32, device="cuda")
    qkv = torch.randn(B, (Hq + 2 * Hkv) * D, device="cuda", generator=g).bfloat16()
    q = ubp.ubp_rotate_append(qkv, Hq, k, v, table, lengths, rotation=ubp.rotation_table(160, D))
    a = ubp.ubp_attention(q, k, v, table, lengths).double()
    b = ubp.ubp_prefix_attention(q, k, v, table, lengths, prefix).double()
    size = v.double().abs().max()
    assert ((a - b).abs() <= 2 * 2.0 ** -8 * a.abs() + 2.0 ** -8 * size).all() and not torch.equal(a, torch.zeros_like(a))
