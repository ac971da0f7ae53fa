"""Token-major products with a block-pruned weight against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from linear_ref import F8, TINY, UNIT, act64, make_weight, product64, quantise, typed_weight

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
IDS = {BF16: "bf16", F16: "f16", F8: "e4m3", F32: "f32"}


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def inputs(T, C, dtype, pad, lead, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(T, C, device="cuda", generator=g)
    xs = None
    if dtype == F8:
        v, xs = quantise(v) if T else (v.to(F8), torch.empty(0, device="cuda"))
    buf = torch.full((T * (C + pad) + lead,), 1.0e4 if dtype != F8 else 448.0, device="cuda").to(dtype)
    x = buf[lead:].view(T, C + pad)[:, :C]
    x.copy_(v.to(dtype))
    return x, xs


def check(ubp, W, mask, Nb, T, dtype, out_dtype, act="none", gated=False, bias=True, residual=True, pad=0, lead=0, seed=0, ypad=0):
    M, C = W.shape
    F = M // 2 if gated else M
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, Nb), dtype, gated=gated)
    x, xs = inputs(T, C, dtype, pad, lead, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    b = torch.randn(M, device="cuda", generator=g) if bias else None
    ybuf = torch.full((T * (F + ypad) + lead,), 7.0, device="cuda", dtype=out_dtype)
    y = ybuf[lead:].view(T, F + ypad)[:, :F]
    r = None
    if residual:
        rbuf = torch.full((T, F + pad), float("nan"), device="cuda", dtype=out_dtype)
        r = rbuf[:, :F]
        r.copy_(torch.randn(T, F, device="cuda", generator=g))
    ubp.ubp_linear(plan, x, bias=b, activation=act, residual=r, x_scales=xs, out=y)
    plan.check()
    x64 = x.double() * (xs.double()[:, None] if xs is not None else 1.0)
    W64 = typed_weight(W, dtype).cuda()
    want, d = product64(x64, W64, None if b is None else b.double(), act, gated, None if r is None else r.double())
    err = (y.double() - want).abs()
    bound = d + UNIT[out_dtype] * (want.abs() + d) + TINY[out_dtype]
    assert torch.isfinite(y.float()).all()
    assert (err <= bound).all(), float((err / bound).max())
    if ypad:
        assert (ybuf[lead:].view(T, F + ypad)[:, F:] == 7.0).all()
    return plan, x, xs, b, r, y


#: (tokens, rows, input features, block rows, sparsity)
SHAPES = [(1, 1, 1, 1, 0), (1, 64, 64, 4, 50), (3, 66, 37, 5, 40), (2, 130, 1003, 2, 70), (4, 258, 515, 8, 80), (8, 300, 2050, 16, 60),
          (9, 96, 129, 3, 50), (5, 1000, 4100, 4, 90), (7, 40, 9000, 4, 50), (23, 260, 512, 4, 70), (64, 128, 64, 2, 50),
          (127, 256, 65, 4, 60), (128, 254, 128, 4, 60), (129, 514, 200, 8, 70), (300, 770, 1000, 4, 80), (513, 32, 1030, 4, 50),
          (2100, 2050, 520, 8, 70), (2600, 4100, 96, 4, 60), (5000, 1030, 70, 2, 50), (40000, 66, 130, 2, 50)]


@pytest.mark.parametrize("dtype", [BF16, F16, F8], ids=IDS.get)
@pytest.mark.parametrize("T,M,C,Nb,p", SHAPES)
def test_product(ubp, dtype, T, M, C, Nb, p):
    W, mask = make_weight(M, C, Nb, p, 100 + M)
    out = BF16 if dtype == F8 else dtype
    check(ubp, W, mask, Nb, T, dtype, out)
    check(ubp, W, mask, Nb, T, dtype, out, act="gelu", residual=False, pad=3, ypad=5, seed=5)
    check(ubp, W, mask, Nb, T, dtype, F32, bias=False, residual=False, pad=8, seed=9)
    if M % 2 == 0:
        check(ubp, W, mask, Nb, T, dtype, out, act="silu", gated=True, bias=False, residual=False, seed=13)
        check(ubp, W, mask, Nb, T, dtype, F32, act="gelu_tanh", gated=True, pad=1, lead=1, ypad=3, seed=17)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T", [1, 6, 150, 40000])
def test_activations(ubp, act, T):
    W, mask = make_weight(96, 80, 4, 50, 3)
    for gated in (False, True):
        for dtype, out in ((BF16, BF16), (F16, F16), (F8, F16), (F8, F32)):
            check(ubp, W, mask, 4, T, dtype, out, act=act, gated=gated, seed=21)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T", [1, 40, 300, 40000])
def test_activations_at_the_ends_of_the_range(ubp, act, T):
    """Arguments up to the largest finite ones, +infinity and NaN (handed in as biases): 0 far below, v far above, NaN stays NaN."""
    a = [1e-30, 1e-3, 0.7, 3.0, 5.5, 9.0, 13.0, 50.0, 86.0, 87.5, 89.0, 200.0, 1e4, 1e20, 3e38]
    v = torch.tensor([0.0] + a + [-k for k in a] + [float("inf"), float("nan")], device="cuda")
    M = v.numel() + 1
    W, mask = make_weight(M, 64, 4, 50, 5)
    b = torch.cat([v, v.new_zeros(1)])
    x = torch.zeros(T, 64, device="cuda", dtype=F16)
    y = ubp.ubp_linear(ubp.LinearPlan(ubp.ubp_pack(W, mask, 4), F16), x, bias=b, activation=act, out=torch.empty(T, M, device="cuda"))
    v64 = b.double()
    want = act64(v64, act)
    if act != "none":
        want = torch.where(v64 < -80, torch.zeros_like(want), want)
    d = 2.0 ** -18 * torch.where(v64 < -80, v64.new_tensor(1e-20), v64.abs()) if act != "none" else torch.zeros_like(want)
    got = y.double()
    assert got[:, v.numel() - 1].isnan().all() and (got[:, v.numel() - 2] == float("inf")).all()
    f = torch.isfinite(v64)
    assert ((got - want)[:, f].abs() <= d[f]).all()


@pytest.mark.parametrize("T", [1, 4, 70, 300, 40000])
def test_rows_without_blocks(ubp, T):
    W, mask = make_weight(64, 48, 4, 95, 3)
    W, mask = W.copy(), mask.copy()
    W[:40], mask[:40] = 0, 0                       # whole output rows empty
    mask[40:] = 0
    mask[44:48, :] = 1                             # and one full stripe
    W = np.where(mask, np.random.default_rng(0).standard_normal(W.shape), 0).astype(np.float32)
    for dtype in (BF16, F8):
        check(ubp, W, mask, 4, T, dtype, BF16, seed=2)
        check(ubp, W, mask, 4, T, dtype, BF16, act="silu", gated=True, seed=3)
    empty = np.zeros_like(mask)
    check(ubp, W * 0, empty, 4, T, F16, F16, act="relu", seed=4)


@pytest.mark.parametrize("T", [1, 3, 40, 260, 9000])
def test_same_result_twice_and_in_place_residual(ubp, T):
    W, mask = make_weight(512, 1500, 4, 70, 8)
    plan, x, xs, b, r, y = check(ubp, W, mask, 4, T, BF16, BF16, seed=30)
    again = ubp.ubp_linear(plan, x, bias=b, residual=r, x_scales=xs)
    assert torch.equal(again, y)
    z = r.contiguous().clone()
    assert ubp.ubp_linear(plan, x, bias=b, residual=z, x_scales=xs, out=z) is z
    assert torch.equal(z, y)


@pytest.mark.parametrize("T", [3, 200, 19500])
def test_bad_token_stays_alone(ubp, T):
    """A NaN or an infinity in one token's row leaves the other tokens' outputs as they are."""
    W, mask = make_weight(256, 300, 4, 60, 8)
    plan, x, xs, b, r, y = check(ubp, W, mask, 4, T, BF16, BF16, seed=31)
    x = x.clone()
    x[1, 7] = float("nan")
    got = ubp.ubp_linear(plan, x, bias=b, residual=r)
    keep = [t for t in range(T) if t != 1]
    assert torch.equal(got[keep], y[keep])
    touched = torch.from_numpy(mask[:, 7] != 0).cuda()
    assert got[1][touched].isnan().all()


@pytest.mark.parametrize("pad", [0, 1])
def test_outputs_on_a_given_stream(ubp, pad):
    """A call on a given stream takes its outputs' (and its workspace's) memory from that stream: a block that the current
    stream has freed may still be written there."""
    W, mask = make_weight(1024, 1536, 4, 60, 8)
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 4), BF16)
    x = inputs(300, 1536, BF16, pad, 0, 5)[0]
    gamma = torch.ones(1536, device="cuda", dtype=BF16)
    calls = [lambda st: ubp.ubp_linear(plan, x, stream=st), lambda st: ubp.ubp_rmsnorm(x, gamma, stream=st)[0],
             lambda st: ubp.ubp_quant_rows(x, stream=st)[0]]
    st = torch.cuda.Stream()
    for call in calls:
        want = call(None)
        torch.cuda.synchronize()
        busy = [torch.empty(n, device="cuda", dtype=torch.uint8) for n in (want.nbytes, 300 * 1536 * 2)]
        torch.cuda._sleep(20_000_000)                # some ten milliseconds, after which the freed blocks are written
        for b in busy:
            b.fill_(0xff)
        del busy, b
        got = call(st)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("T", [2, 100])
def test_other_stream_and_no_tokens(ubp, T):
    W, mask = make_weight(256, 320, 4, 60, 8)
    plan, x, xs, b, r, y = check(ubp, W, mask, 4, T, F16, F16, pad=1, seed=32)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        z = x
        for _ in range(20):
            z = z * 1.0
        got = ubp.ubp_linear(plan, z, bias=b, residual=r)
    st.synchronize()
    assert torch.equal(got, y)
    got = ubp.ubp_linear(plan, x, bias=b, residual=r, stream=st)
    st.synchronize()
    assert torch.equal(got, y)
    assert ubp.ubp_linear(plan, x[:0]).shape == (0, 256) and plan.choice(0) == plan.choice(1)


def test_row_scales(ubp):
    W, mask = make_weight(70, 90, 2, 60, 4)
    W[3], mask[3] = W[3], mask[3]
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 2), F8)
    assert torch.equal(plan.row_scales.cpu(), quantise(torch.from_numpy(W))[1])
    assert ubp.LinearPlan(ubp.ubp_pack(W, mask, 2), BF16).row_scales is None


def test_block_of_a_feed_forward_layer(ubp):
    """Norm -> gated product -> rows to 8 bits -> product with the residual, each step against 64 bits from the step's
    own inputs."""
    C, F, T = 256, 640, 37
    Wg, mg = make_weight(2 * F, C, 4, 70, 1)
    Wd, md = make_weight(C, F, 4, 70, 2)
    up, down = ubp.LinearPlan(ubp.ubp_pack(Wg, mg, 4), F8, gated=True), ubp.LinearPlan(ubp.ubp_pack(Wd, md, 4), F8)
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r = (torch.randn(T, C, device="cuda", generator=g).to(BF16) for _ in range(2))
    q, s, h = ubp.ubp_rmsnorm(x, torch.ones(C, device="cuda", dtype=BF16), 1e-5, residual=r, out_dtype=F8)
    a = ubp.ubp_linear(up, q, activation="silu", x_scales=s)
    want, d = product64(q.double() * s.double()[:, None], typed_weight(Wg, F8).cuda(), None, "silu", True, None)
    assert ((a.double() - want).abs() <= d + UNIT[BF16] * (want.abs() + d)).all()
    p, ps = ubp.ubp_quant_rows(a)
    y = ubp.ubp_linear(down, p, residual=h, x_scales=ps, out=h.clone())
    want, d = product64(p.double() * ps.double()[:, None], typed_weight(Wd, F8).cuda(), None, "none", False, h.double())
    assert ((y.double() - want).abs() <= d + UNIT[BF16] * (want.abs() + d)).all()


def test_refusals(ubp):
    W, mask = make_weight(64, 32, 4, 50, 1)
    blob = ubp.ubp_pack(W, mask, 4)
    plan, p8 = ubp.LinearPlan(blob, BF16), ubp.LinearPlan(blob, F8)
    x = torch.randn(4, 32, device="cuda").to(BF16)
    s = torch.ones(4, device="cuda")
    bad = [lambda: ubp.ubp_linear(plan, x.half()), lambda: ubp.ubp_linear(plan, x[:, :31]), lambda: ubp.ubp_linear(plan, x, x_scales=s),
           lambda: ubp.ubp_linear(p8, x.to(F8)), lambda: ubp.ubp_linear(plan, x, activation="swish"),
           lambda: ubp.ubp_linear(plan, x, bias=torch.zeros(63, device="cuda")), lambda: ubp.ubp_linear(plan, x, bias=torch.zeros(64, device="cuda").half()),
           lambda: ubp.ubp_linear(plan, x, residual=torch.zeros(4, 64, device="cuda")), lambda: ubp.ubp_linear(plan, x.cpu()),
           lambda: ubp.ubp_linear(plan, x, out=torch.zeros(4, 63, device="cuda", dtype=BF16)),
           lambda: ubp.ubp_linear(plan, x[:1].expand(4, 32)), lambda: ubp.LinearPlan(blob, F32)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f, code in ((lambda: ubp.ubp_linear(plan, x, out_dtype=F16), -1),
                    (lambda: ubp.ubp_linear(p8, x.to(F8), x_scales=s, out_dtype=F8), -1),
                    (lambda: ubp.LinearPlan(blob[:-1], BF16), -4)):
        with pytest.raises(ubp.UbpError) as e:
            f()
        assert e.value.code == code
    W1, m1 = make_weight(33, 32, 1, 50, 1)
    with pytest.raises(ubp.UbpError):
        ubp.LinearPlan(ubp.ubp_pack(W1, m1, 1), BF16, gated=True)          # an odd number of rows has no halves
    plan.free()
    with pytest.raises(RuntimeError):
        ubp.ubp_linear(plan, x)


#: (tokens, rows, input features, block rows, sparsity, what the call has to take): every kernel and tile,
#: (0, tokens a block), (1, tokens of a tile, parts of the reduction), (2, rows of a tile)
PATHS = [(1, 2048, 2048, 4, 0, (0, 1)), (2, 2048, 2048, 4, 60, (0, 2)), (3, 2048, 2048, 4, 80, (0, 4)), (8, 2048, 2048, 4, 90, (0, 8)),
         (1, 9000, 6000, 2, 70, (0, 1)), (1, 6000, 6000, 8, 70, (0, 1)), (1, 400, 50000, 2, 50, (0, 1)), (2, 9000, 6000, 4, 70, (0, 2)), (4, 6000, 6000, 8, 70, (0, 4)),
         (16, 512, 512, 8, 95, (0, 8)), (16, 2048, 2048, 4, 0, (1, 16, 4)), (20, 300, 3000, 2, 70, (1, 32, 8)), (77, 4000, 260, 4, 70, (1, 48, 1)),
         (256, 130, 600, 4, 70, (1, 64, 4)), (257, 130, 600, 4, 70, (1, 64, 4)), (777, 770, 1000, 4, 70, (1, 80, 2)), (1000, 4000, 260, 4, 70, (1, 256, 1)),
         (2600, 1030, 70, 2, 60, (1, 176, 1)), (5000, 300, 3000, 4, 70, (1, 224, 2)), (2100, 4100, 96, 4, 80, (2, 128)), (5000, 1030, 70, 2, 60, (2, 128)),
         (2100, 2048, 2048, 4, 60, (2, 256)), (9000, 770, 1000, 4, 60, (2, 256))]


@pytest.mark.parametrize("T,M,C,Nb,p,path", PATHS)
def test_every_kernel(ubp, T, M, C, Nb, p, path):
    W, mask = make_weight(M, C, Nb, p, 7 * M + C)
    for dtype, out in ((BF16, BF16), (F16, F32), (F8, BF16)):
        plan = check(ubp, W, mask, Nb, T, dtype, out, pad=8, seed=41)[0]
        if dtype == BF16:
            assert plan.choice(T)[:len(path)] == path
        check(ubp, W, mask, Nb, T, dtype, out, act="silu", gated=True, residual=False, seed=43)


@pytest.mark.parametrize("ypad,rpad", [(0, 0), (4, 4), (2, 2), (1, 1), (8, 2), (0, 8)])
def test_output_alignments(ubp, ypad, rpad):
    """Rows of y and of the residual aligned to 16, 8, 4 and 2 bytes, features a multiple of that or not."""
    for M in (512, 500, 508, 502, 501):
        W, mask = make_weight(M, 96, 1, 60, M)
        for T, out in ((300, BF16), (300, F32), (40, BF16), (2, BF16), (20000, BF16), (20000, F32)):
            check(ubp, W, mask, 1, T, BF16, out, act="relu", pad=rpad, ypad=ypad, seed=51)


def test_offsets_beyond_32_bits(ubp):
    W, mask = make_weight(96, 200, 4, 60, 8)
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 4), BF16)
    for T, ld in ((3, (1 << 30) + 8), (18, (1 << 27) + 8)):
        buf = torch.empty(T * ld, dtype=BF16, device="cuda")
        x = buf.view(T, ld)[:, :200]
        x.copy_(torch.randn(T, 200, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)))
        y = buf.view(T, ld)[:, 1024:1120]
        want = ubp.ubp_linear(plan, x.contiguous())
        ubp.ubp_linear(plan, x, out=y)
        assert torch.equal(y, want)
        del buf, x, y


@pytest.mark.parametrize("T", [1, 5, 30, 300, 5000])
def test_launches_back_to_back(ubp, T):
    """The calls' kernels start before the ones before them have finished: a chain in which every call reads what the call
    before wrote, over buffers that are used again, gives the same values every time."""
    C, F = 512, 1024
    Wg, mg = make_weight(2 * F, C, 4, 80, 1)
    Wd, md = make_weight(C, F, 4, 80, 2)
    up, down = ubp.LinearPlan(ubp.ubp_pack(Wg, mg, 4), F8, gated=True), ubp.LinearPlan(ubp.ubp_pack(Wd, md, 4), F8)
    g = torch.Generator(device="cuda").manual_seed(0)
    x0, h0 = (torch.randn(T, C, device="cuda", generator=g).to(BF16) for _ in range(2))
    gamma = torch.ones(C, device="cuda", dtype=BF16)
    q, s, a = torch.empty(T, C, device="cuda", dtype=F8), torch.empty(T, device="cuda"), torch.empty(T, F, device="cuda", dtype=BF16)
    p, t, h = torch.empty(T, F, device="cuda", dtype=F8), torch.empty(T, device="cuda"), torch.empty_like(h0)

    def chain(sync):
        h.copy_(h0)
        for _ in range(6):
            for call in (lambda: ubp.ubp_rmsnorm(x0, gamma, 1e-5, residual=h, residual_out=h, out=q, scales=s),
                         lambda: ubp.ubp_linear(up, q, activation="silu", x_scales=s, out=a),
                         lambda: ubp.ubp_quant_rows(a, out=p, scales=t),
                         lambda: ubp.ubp_linear(down, p, residual=h, x_scales=t, out=h)):
                call()
                if sync:
                    torch.cuda.synchronize()
        return h.clone()

    want = chain(True)
    assert torch.isfinite(want.float()).all()
    for _ in range(20):
        assert torch.equal(chain(False), want)
    up.check()
    down.check()


def test_example_runs():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "pruned_feed_forward.py"), "--width", "512", "--hidden", "1024"],
                       cwd=root, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "pruned feed-forward ok" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


def test_checked_build():
    """The same cases on the checked build of the library, whose kernels compare the plan's indices with their extents."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lib = os.path.join(root, "paper_2407_19644_b200", "libubp_b200_debug.so")
    if not os.path.exists(lib):
        from paper_2407_19644_b200 import build
        build.build(debug=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_linear.py", "tests/test_gpu_rows.py", "-q", "-x", "-m", "gpu", "-k",
                        "test_product or test_every_kernel or test_rows_without_blocks or test_special"], cwd=root,
                       env=dict(os.environ, UBP_B200_LIBRARY=lib), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
