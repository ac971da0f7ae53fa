"""Damaged plans of the token-major product on the checked build of the library (run as a script with UBP_B200_LIBRARY pointing
at libubp_b200_debug.so). The kept-block kernel has to report, through the plan's status word, a channel index just past the
row (a value the ordinary build would survive too: the activations' padding follows) and a bundle that starts after its end
(nothing is read then), and to run clean again on the plan as it was."""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2407_19644_b200 as ubp  # noqa: E402
from linear_ref import F8, make_weight  # noqa: E402

M, C, Nb = 256, 500, 4
W, mask = make_weight(M, C, Nb, 80, 5)
blob = ubp.ubp_pack(W, mask, Nb)
assert ubp.lib_path().endswith("libubp_b200_debug.so"), ubp.lib_path()


def status(plan, x, xs):
    ubp.ubp_linear(plan, x, x_scales=xs)
    torch.cuda.synchronize()
    at = plan._dev - plan.buffer.data_ptr()
    word = int(plan.buffer[at:at + 4].cpu().numpy().view(np.int32)[0])
    try:
        plan.check()
        assert word == 0
    except ubp.UbpError as e:
        assert e.code == -7 and word != 0
    plan.clear_status()
    return word


for dtype in (torch.bfloat16, torch.float16, F8):
    img, geom, offs = ubp.linear_plan_image(blob, dtype)
    plan = ubp.LinearPlan(blob, dtype)
    base = plan._dev - plan.buffer.data_ptr()
    idx = plan.buffer[base + offs["idx"]:base + offs["idx"] + 2].view(torch.int16)
    off = plan.buffer[base + offs["off"]:base + offs["off"] + 8].view(torch.int32)
    for T in (1, 2, 3, 8):
        assert plan.choice(T)[0] == 0
        x = torch.randn(T, C, device="cuda").to(dtype)
        xs = torch.ones(T, device="cuda") if dtype == F8 else None
        assert status(plan, x, xs) == 0
        for view, at, bad in ((idx, 0, C), (off, 0, int(off[1]) + 1)):
            was = view[at].clone()
            view[at] = bad
            assert status(plan, x, xs) == 2, (dtype, T, bad)
            view[at] = was
        assert status(plan, x, xs) == 0
    print(f"{dtype}: damaged plan noticed")
print("checked linear ok")
