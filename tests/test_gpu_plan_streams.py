"""Plans built on a given stream, used on streams other than their own, and dropped while calls are still pending."""
import pytest
import torch

from linear_ref import F8, make_weight

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
LONG = 20_000_000                # clock cycles of a pause on the GPU: some ten milliseconds


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def leave_writes_pending(nbytes):
    """Blocks of about this size that the current stream has freed and will still write to."""
    busy = [torch.empty(n, device="cuda", dtype=torch.uint8) for n in (nbytes, nbytes, nbytes)]
    torch.cuda._sleep(LONG)
    for b in busy:
        b.zero_()


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
def test_linear_plan_built_on_a_given_stream(ubp, dtype):
    """The plan's memory comes from the stream that uploads it, so nothing that the current stream has yet to write reaches it."""
    W, mask = make_weight(1024, 1536, 4, 60, 8)
    blob = ubp.ubp_pack(W, mask, 4)
    want = torch.from_numpy(ubp.linear_plan_image(blob, dtype)[0])
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    leave_writes_pending(want.numel() + 256)
    plan = ubp.LinearPlan(blob, dtype, stream=st)
    torch.cuda.synchronize()
    at = plan._dev - plan.buffer.data_ptr()
    assert torch.equal(plan.buffer[at:at + want.numel()].cpu(), want)


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("given", [False, True])
def test_linear_plan_dropped_while_another_stream_uses_it(ubp, T, given):
    """A call on another stream than the plan's keeps the plan's memory until it has run (a zeroed plan would give zeros)."""
    W, mask = make_weight(1024, 1536, 4, 60, 8)
    blob = ubp.ubp_pack(W, mask, 4)
    x = torch.randn(T, 1536, device="cuda").to(BF16)
    plan = ubp.LinearPlan(blob, BF16)
    want, n = ubp.ubp_linear(plan, x), plan.buffer.numel()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(LONG)
        if not given:
            got = ubp.ubp_linear(plan, x)
    if given:
        got = ubp.ubp_linear(plan, x, stream=st)
    del plan
    for _ in range(3):
        torch.empty(n, device="cuda", dtype=torch.uint8).zero_()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_image_plan_and_outputs_on_a_given_stream(ubp):
    """The same for the plans and calls on images: plan, outputs and scratch belong to the stream that writes them."""
    import numpy as np
    import ubp_synth
    L = ubp_synth.make_layer("streams", 256, 512, 4, 70, 3, Nc=64)
    blob = ubp.ubp_pack(L.W, L.mask, 4)
    st = torch.cuda.Stream()
    plan = ubp.Plan(blob)
    want = torch.from_numpy(ubp.plan_image(blob, plan.variant)[0])
    torch.cuda.synchronize()
    leave_writes_pending(plan.buffer.numel())
    late = ubp.Plan(blob, stream=st)
    torch.cuda.synchronize()
    at = late._dev - late.buffer.data_ptr()
    assert torch.equal(late.buffer[at:at + want.numel()].cpu(), want)
    x = torch.randn(512, 4, 32, 32, device="cuda")
    r = ubp_synth.make_layer("streams", 64, 64, 4, 70, 4, B=2, H=32, Wd=32, R=9)
    p3, x3 = ubp.Plan(ubp.ubp_pack(r.W, r.mask, 4)), torch.from_numpy(r.X).cuda()
    W = torch.from_numpy(np.ascontiguousarray(L.W[:, :, 0])).cuda()
    calls = [lambda s: ubp.ubp_spmm(plan, x.view(512, -1), stream=s), lambda s: ubp.ubp_conv1x1(plan, x, stream=s),
             lambda s: ubp.ubp_conv1x1(plan, x, stride=2, stream=s), lambda s: ubp.ubp_conv3x3_implicit(p3, x3, stream=s),
             lambda s: ubp.ubp_conv3x3_implicit(p3, x3, stride=2, stream=s), lambda s: ubp.ubp_block_scores(W, 4, stream=s),
             lambda s: ubp.ubp_bed_select(W, 4, 500, stream=s)[0], lambda s: ubp.ubp_bed_select(W, 4, 500, stream=s)[1]]
    for call in calls:
        want = call(None)
        torch.cuda.synchronize()
        leave_writes_pending(want.nbytes)
        got = call(st)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_image_plan_dropped_while_another_stream_uses_it(ubp):
    import ubp_synth
    L = ubp_synth.make_layer("streams", 256, 512, 4, 70, 3, Nc=64)
    blob = ubp.ubp_pack(L.W, L.mask, 4)
    x = torch.randn(512, 4096, device="cuda")
    for given in (False, True):
        plan = ubp.Plan(blob)
        want, n = ubp.ubp_spmm(plan, x), plan.buffer.numel()
        st = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            torch.cuda._sleep(LONG)
            if not given:
                got = ubp.ubp_spmm(plan, x)
        if given:
            got = ubp.ubp_spmm(plan, x, stream=st)
        del plan
        for _ in range(3):
            torch.empty(n, device="cuda", dtype=torch.uint8).zero_()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
def test_two_streams_use_one_plan_at_once(ubp, dtype):
    W, mask = make_weight(2048, 1024, 4, 70, 8)
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 4), dtype)
    sizes = [1, 3, 24, 200, 2500]
    xs = [torch.randn(T, 1024, device="cuda").to(dtype) for T in sizes]
    sc = [torch.ones(T, device="cuda") if dtype == F8 else None for T in sizes]
    want = [ubp.ubp_linear(plan, x, x_scales=s) for x, s in zip(xs, sc)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for k, st in enumerate(streams):
            order = range(len(sizes)) if k == 0 else reversed(range(len(sizes)))
            with torch.cuda.stream(st):
                got[k] += [(i, ubp.ubp_linear(plan, xs[i], x_scales=sc[i])) for i in order]
    torch.cuda.synchronize()
    plan.check()
    for i, y in got[0] + got[1]:
        assert torch.equal(y, want[i])


def test_two_threads_use_one_plan_at_once(ubp):
    """Through the C entry point, which ctypes calls without the interpreter's lock; the kernels' first calls among them."""
    import threading
    W, mask = make_weight(2048, 1024, 2, 70, 8)
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 2), torch.float16)
    sizes = [1, 2, 5, 24, 200, 2500]
    x = [torch.randn(T, 1024, device="cuda").half() for T in sizes]
    L, failed = ubp.load(), []
    out = [[torch.empty(T, 2048, device="cuda", dtype=torch.float16) for T in sizes] for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]

    def work(k):
        torch.cuda.set_device(0)
        for _ in range(20):
            for i, T in enumerate(sizes):
                rc = L.ubp_linear(plan.handle, x[i].data_ptr(), 1024, None, T, None, 0, None, 0, out[k][i].data_ptr(), 2048, 1, None, 0,
                                  streams[k].cuda_stream)
                if rc:
                    failed.append(rc)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    plan.check()
    assert not failed
    for i in range(len(sizes)):
        want = ubp.ubp_linear(plan, x[i])
        assert torch.equal(out[0][i], want) and torch.equal(out[1][i], want)


@pytest.mark.parametrize("T", [1, 8, 40, 300, 5000])
@pytest.mark.parametrize("pad", [0, 1])
def test_calls_are_captured_into_a_graph(ubp, T, pad):
    """A feed-forward block as one graph: replays read the inputs as they are then and give the values of plain calls."""
    C, F = 512, 1024
    Wg, mg = make_weight(2 * F, C, 4, 80, 1)
    Wd, md = make_weight(C, F, 4, 80, 2)
    up, down = ubp.LinearPlan(ubp.ubp_pack(Wg, mg, 4), F8, gated=True), ubp.LinearPlan(ubp.ubp_pack(Wd, md, 4), BF16)
    gamma = torch.ones(C, device="cuda", dtype=BF16)
    x = torch.randn(T, C + pad, device="cuda").to(BF16)[:, :C]
    r = torch.randn(T, C, device="cuda").to(BF16)

    def block():
        q, s, h = ubp.ubp_rmsnorm(x, gamma, 1e-5, residual=r, out_dtype=F8)
        a = ubp.ubp_linear(up, q, activation="silu", x_scales=s)
        b = torch.empty(T, F + pad, device="cuda", dtype=BF16)[:, :F]
        b.copy_(a)
        p, t = ubp.ubp_quant_rows(b)
        return ubp.ubp_linear(down, b, residual=h), p, t

    block()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = block()
    for seed in range(3):
        x.copy_(torch.randn(T, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        g.replay()
        want = block()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.float(), b.float())
    up.check()
    down.check()
