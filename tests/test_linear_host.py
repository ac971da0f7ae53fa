"""Plan image of the token-major products and the C entry points' checks, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2407_19644_b200 as ubp
from linear_ref import F8, make_weight, quantise

DT = {torch.float16: 1, torch.bfloat16: 2, F8: 3}


def replay(img, geom, offs, M, C, mask_at):
    """The image's sparse entries scattered into a dense [M][C] array of codes, and how often each place was written."""
    nbk, epc, b, lanes = geom["nbk"], geom["epc"], geom["bytes"], geom["lanes"]
    rb = 32 // lanes
    assert nbk * epc * b == 16 and lanes in (8, 16, 32)
    nb = -(-M // rb)
    off = np.frombuffer(img, "<u4", nb + 1, offs["off"])
    n = int(off[-1])
    idx = np.frombuffer(img, "<u2", n * 32 * epc, offs["idx"]).reshape(n, rb, lanes * epc)
    val = np.frombuffer(img, "<u2" if b == 2 else "u1", n * 32 * epc * nbk, offs["val"]).reshape(n, rb, lanes * epc, nbk)
    out, hits = np.zeros((M, C), val.dtype), np.zeros((M, C), np.int32)
    assert off[0] == 0 and (np.diff(off.astype(np.int64)) >= 0).all()
    for i in range(nb * rb):
        q, u = divmod(i, rb)
        js, ws = idx[off[q]:off[q + 1], u].reshape(-1), val[off[q]:off[q + 1], u].reshape(-1, nbk)
        seen = set()
        for e, j in enumerate(js.tolist()):
            assert j < C
            if i >= M or j in seen or not (i + nbk <= M and mask_at(i, j)):   # a filler: the row's last channel again, weight zero
                assert not ws[e].any() and (j == js[e - 1] if e and seen else j == 0)
                continue
            seen.add(j)
            out[i:i + nbk, j] = ws[e]
            hits[i:i + nbk, j] += 1
    return out, hits


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F8], ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("M,C,Nb,p,gated", [(1, 1, 1, 0, False), (64, 600, 4, 60, False), (66, 37, 5, 40, True), (50, 1100, 16, 70, True),
                                            (34, 4097, 6, 50, True), (130, 512, 2, 80, False), (40, 8200, 4, 80, True), (32, 20, 8, 100, True)])
def test_plan_image_holds_the_weight(dtype, M, C, Nb, p, gated):
    W, mask = make_weight(M, C, Nb, p, 5)
    img, geom, offs = ubp.linear_plan_image(ubp.ubp_pack(W, mask, Nb), dtype, gated)
    if dtype == F8:
        q, s = quantise(torch.from_numpy(W))
        want = q.view(torch.uint8).numpy() * (mask != 0)
        assert np.array_equal(np.frombuffer(img, "<f4", M, offs["scale"]), s.numpy())
    else:
        want = torch.from_numpy(W).to(dtype).view(torch.int16).numpy().view(np.uint16) * (mask != 0)
    # start rows of the entries: the blocks' own, and every nbk rows inside them
    v = ubp.blob_view(ubp.ubp_pack(W, mask, Nb))
    starts = {(i + s, int(j)) for i in range(M) for j in v["indices"][v["indptr"][i]:v["indptr"][i + 1]] for s in range(0, Nb, geom["nbk"])}
    got, hits = replay(img, geom, offs, M, C, lambda i, j: (i, j) in starts)
    assert np.array_equal(hits, (mask != 0).astype(np.int32))
    assert np.array_equal(got, want)
    Mp, Kp, b = geom["Mp"], geom["Kp"], geom["bytes"]
    assert Mp % 128 == 0 and Kp * b % 128 == 0 and Kp >= C
    dense = np.frombuffer(img, want.dtype, Mp * Kp, offs["dense"]).reshape(Mp, Kp)
    expect = np.zeros_like(dense)
    if gated:
        for f in range(M // 2):
            expect[f // 16 * 32 + f % 16, :C] = want[f]
            expect[f // 16 * 32 + 16 + f % 16, :C] = want[M // 2 + f]
    else:
        expect[:M, :C] = want
    assert np.array_equal(dense, expect)
    assert not np.frombuffer(img, np.uint8, 256).any()


def test_block_rows_per_entry():
    for Nb, nbk in ((1, 1), (2, 2), (3, 1), (4, 4), (6, 2), (8, 8), (12, 4), (16, 8)):
        W, mask = make_weight(48, 16, Nb, 50, 1)
        assert ubp.linear_plan_image(ubp.ubp_pack(W, mask, Nb), torch.bfloat16)[1]["nbk"] == nbk


def test_c_entry_refusals():
    """Bad arguments come back as status codes before anything touches a device."""
    L = ubp.load()
    W, mask = make_weight(32, 16, 4, 50, 1)
    blob = np.frombuffer(ubp.ubp_pack(W, mask, 4), np.uint8)
    ptr, n = blob.ctypes.data, ctypes.c_size_t(0)
    assert L.ubp_linear_plan_size(ptr, blob.size, 2, 0, ctypes.byref(n)) == 0 and n.value > 0
    assert L.ubp_linear_plan_size(ptr, blob.size, 0, 0, ctypes.byref(n)) == -1            # fp32 is no plan type
    assert L.ubp_linear_plan_size(ptr, blob.size, 7, 0, ctypes.byref(n)) == -1
    assert L.ubp_linear_plan_size(ptr, blob.size, 2, 0, None) == -1
    assert L.ubp_linear_plan_size(ptr, blob.size - 1, 2, 0, ctypes.byref(n)) == -4
    W9 = np.random.default_rng(0).standard_normal((32, 4, 9)).astype(np.float32)
    b9 = np.frombuffer(ubp.ubp_pack(W9, np.ones((32, 4), np.uint8), 4), np.uint8)
    assert L.ubp_linear_plan_size(b9.ctypes.data, b9.size, 2, 0, ctypes.byref(n)) == -6   # 3x3 taps
    p = 1 << 20                                                                           # (never dereferenced)
    h = ctypes.c_void_p()
    assert L.ubp_linear_plan_build(ptr, blob.size, 2, 0, p + 8, 1 << 30, None, ctypes.byref(h)) == -1     # alignment
    assert L.ubp_linear_plan_build(ptr, blob.size, 2, 0, p, 100, None, ctypes.byref(h)) == -3
    assert L.ubp_linear(None, p, 16, None, 1, None, 0, None, 0, p, 32, 2, None, 0, None) == -1
    assert L.ubp_linear_plan_check(None, None) == -1
    ok = [p, 64, p, 64, p, 2, 2, 4, 64, 1e-5, p, 64, p, 64, 2, p, None]
    for at, v in ((0, None), (1, 63), (3, 63), (4, None), (5, 1), (6, 3), (6, 9), (7, -1), (8, 0), (9, -1.0), (9, float("nan")),
                  (11, 63), (12, None), (13, 63), (14, 1), (0, p + 1), (12, p + 1)):
        a = list(ok)
        a[at] = v
        assert L.ubp_rmsnorm(*a) == -1, (at, v)
    a = list(ok)
    a[14], a[15] = 3, None
    assert L.ubp_rmsnorm(*a) == -1                                                        # 8-bit rows without scales
    a = list(ok)
    a[7] = 0
    assert L.ubp_rmsnorm(*a) == 0                                                         # no rows: nothing to do
    ok = [p, 64, 2, 4, 64, p, 64, p, None]
    for at, v in ((0, None), (1, 63), (2, 3), (3, -1), (4, 0), (5, None), (6, 63), (7, None), (7, p + 2)):
        a = list(ok)
        a[at] = v
        assert L.ubp_quant_rows(*a) == -1, (at, v)


def test_c_entry_refuses_outputs_over_inputs():
    L, p, q = ubp.load(), 1 << 20, 1 << 21                                                # (never dereferenced)
    ok = [p, 64, None, 0, q, 2, 2, 4, 64, 1e-5, None, 64, p + 4096, 64, 2, None, None]
    for changes in ({2: p + 8192, 3: 64, 10: p + 4096}, {10: p, 11: 72}, {2: p + 8192, 3: 64, 10: p + 8192, 11: 72}):
        a = list(ok)
        for at, v in changes.items():
            a[at] = v
        assert L.ubp_rmsnorm(*a) == -1, changes
