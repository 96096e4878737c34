"""Bounded waits of the 8-bit head's product: they run out, are reported, and the kernel ends by itself."""
import pytest
import torch

import test_gpu_beams as beams
from paper_2405_04304_b200 import binding
from test_gpu_beams import I32, beam_scores, context, gen, head, logits_of, randn

pytestmark = pytest.mark.gpu


# rows rounded in the kernel; one block of vocabulary rows to a CTA, two blocks, pairs of CTAs
@pytest.mark.parametrize("V,d,R", [(4000, 256, 4), (4000, 256, 24), (4000, 256, 100), (40011, 1000, 100), (5000, 2048, 257)])
def test_waits_of_a_product_that_run_out_are_reported_and_nothing_hangs(V, d, R):
    g = gen(V + R)
    Wq, ws = head(V, d, g)
    H, score = randn(g, R, d).bfloat16(), beam_scores(g, R, 1)
    y, work = torch.zeros((R, V), device="cuda"), torch.zeros((R, V), device="cuda")
    s, p, t = torch.zeros((R, 1), device="cuda"), torch.zeros((R, 1), dtype=I32, device="cuda"), torch.zeros((R, 1), dtype=I32, device="cuda")
    want = logits_of(Wq, ws, H)
    good = context(V, d, batch=R, rows=R)
    good.project_int8(Wq, ws, H, y)
    assert torch.equal(y, want) and good.device_status() == 0
    ctx = context(V, d, batch=R, rows=R)
    ctx.test_hooks(wait_budget_clocks=2_000_000, withhold_records=True)      # about a millisecond
    try:
        ctx.project_int8(Wq, ws, H, y)
        assert ctx.device_status() == binding.ERR_TIMEOUT                    # (the kernel has ended by itself)
        assert ctx.device_status() == 0
        ctx.beam_step_int8(Wq, ws, H, score, s, p, t, work)
        assert ctx.device_status() == binding.ERR_TIMEOUT
    finally:
        ctx.test_hooks(0, False)                                             # default budget again
        ctx.close()
    for again in (good, context(V, d, batch=R, rows=R)):                     # other contexts are not affected
        y.zero_()
        again.project_int8(Wq, ws, H, y)
        assert torch.equal(y, want) and again.device_status() == 0
        again.beam_step_int8(Wq, ws, H, score, s, p, t, work)
        assert torch.equal(work, want) and torch.equal(t.cpu().long()[:, 0], want.argmax(1).cpu()) and (p == 0).all()
        assert again.device_status() == 0
