"""Selections at the edges of what the arithmetic holds: masks of any size, and logits and scores as large as fp32 has them."""
import math

import pytest
import torch

import test_gpu_beams as beams
from test_gpu_beams import BF16, F16, F32, I32, beam_scores, check_select, gen, head, logits_of, randn

pytestmark = pytest.mark.gpu

MASKS = [-1e5, -1.6e7, -1.7e7, -1e9, -1e10, -1e12, -1e20, -1e30]


# ------------------------------------------------------------------------------------------------ masks and large logits
def masked(g, rows, V, mask, z_type):
    """Logits of which some tokens are not allowed: whole segments of 1024, parts of them, all but one, whole chunks of 32 and of 128."""
    z = randn(g, rows, V)
    z[0, 1024:2048] = mask
    z[1, :2048] = mask
    z[2, 1000:] = mask
    z[3, 1:] = mask
    z[4, 32:64] = mask
    z[5, 128:256] = mask
    z[6, ::2] = mask
    z[7] = mask + 0.0 * z[7]                        # nothing allowed: every token as good as the others
    return z.to(z_type)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("z_type", [F32, BF16])
@pytest.mark.parametrize("B,V", [(2, 5000), (40, 2500)])          # one launch, and two
def test_select_masks_of_any_size(mask, z_type, B, V):
    g = gen(B + V)
    z = torch.cat([masked(g, 8, V, mask, z_type) for _ in range(B // 2)])
    check_select(z, beam_scores(g, B, 4), 6)


@pytest.mark.parametrize("size", [1.6e7, 1.7e7, 1e9, 1e10, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("z_type", [F32, BF16])
def test_select_logits_of_any_size(size, z_type):
    """Rows whose largest logit is far from 0, on either side."""
    g = gen(3)
    z = randn(g, 8, 3000)
    z[0] += size
    z[1] -= size
    z[2, 7] = size
    z[3, 1500] = size
    z[4, 100:1200] -= size
    z[5] *= size
    check_select(z.to(z_type), beam_scores(g, 2, 4), 5)


@pytest.mark.parametrize("size", [1e8, 1e10, 1e12, 1e20, 1e30])
def test_step_logits_of_any_size(size):
    """Vocabulary rows whose scale makes logits of any size, by whole chunks and one by one, on either side of 0."""
    V, d, B, K, n = 3000, 128, 2, 3, 5
    for sign in (-1, 1):
        g = gen(5)
        Wq, ws = head(V, d, g)
        ws *= 5.0
        H = randn(g, B * K, d).bfloat16().abs()
        for rows in (slice(64, 96), slice(1024, 2048), slice(2500, 2501)):
            Wq[rows] = 127 * sign
            ws[rows] = size / (127.0 * d)
        z = logits_of(Wq, ws, H)
        assert float(z.abs().max()) > size / 8 and bool(torch.isfinite(z).all())
        score = beam_scores(g, B, K)
        want_s, want_p, want_t, _, gap = beams.best_of(z, score, n)
        assert gap > 4 * beams.LSE_TOL
        s, p, t = torch.zeros((B, n), device="cuda"), torch.zeros((B, n), dtype=I32, device="cuda"), torch.zeros((B, n), dtype=I32, device="cuda")
        ctx = beams.context(V, d, batch=B, rows=B * K)
        ctx.beam_step_int8(Wq, ws, H, score, s, p, t, torch.empty((B * K, V), device="cuda"))
        assert torch.equal(p.cpu().long(), want_p) and torch.equal(t.cpu().long(), want_t)
        assert ((s.cpu().double() - want_s).abs() <= beams.score_tol(want_s)).all()


# ------------------------------------------------------------------------------------------------ small vocabularies
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 64])
@pytest.mark.parametrize("B,K", [(8, 8), (64, 4), (4, 64)])
def test_select_small_vocabularies_with_every_row_of_the_context(V, B, K):
    """(A row's statistics take more room than one record of the 8-bit head's.)"""
    g = gen(V * 100 + B)
    check_select(randn(g, B * K, V), beam_scores(g, B, K), K)


# ------------------------------------------------------------------------------------------------ scores that come near to each other
def lists_of(ctx, z, score, n):
    B = score.shape[0]
    s, p, t = torch.full((B, n), 7.0, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda")
    ctx.beam_select(z, score, s, p, t)
    assert ctx.device_status() == 0
    return s.cpu().double(), p.cpu().long(), t.cpu().long()


@pytest.mark.parametrize("B", [16, 40])                           # one launch, and two
def test_select_peaked_rows_next_to_zero(B):
    """Two beams with one likely token each, whose scores differ by less than the rounding of a sum of exponentials next to 1.

    Sums 1 + (m + 0.49) u and 1 + (m - 0.49) u with u = 2^-23: in fp32 they are 1 + m u both.  The second beam's score is 0.9 u lower, so its
    token is the better one by 0.08 u, while it looks the worse by 0.9 u.  (A sum's own error is 2^-18 of what it has beyond 1: 2^-13 u.)"""
    V, u = 2048, 2.0 ** -23
    z, score = torch.full((B, 2, V), -math.inf, device="cuda"), torch.zeros((B, 2), device="cuda")
    for b in range(B):
        m = 2 + b
        z[b, :, 3] = 0.0
        z[b, 0, 1500], z[b, 1, 1500] = math.log((m + 0.49) * u), math.log((m - 0.49) * u)
    score[:, 1] = -0.9 * u
    l = score.double().cpu()[:, :, None] + torch.log_softmax(z.double().cpu(), 2)
    assert (l[:, 1, 3] - l[:, 0, 3] > 0.05 * u).all()
    ctx = beams.context(V, batch=B, rows=2 * B)
    s, p, t = lists_of(ctx, z.view(2 * B, V), score, 1)
    assert (p == 1).all() and (t == 3).all()
    s, p, t = lists_of(ctx, z.view(2 * B, V), score, 2)
    assert (p == torch.tensor([1, 0])).all() and (t == 3).all()


@pytest.mark.parametrize("B", [4, 40])                            # one launch, and two
def test_select_offsets_beyond_fp32(B):
    """A beam at -3e38 whose logits are all 3e38: score minus logarithm is beyond fp32, the scores themselves (-3e38) are not, and they are
    better than those of the beam before it.  And the other way round, where the largest logit is far below 0."""
    V, K, n = 1500, 3, 6
    z, score = randn(gen(B), B, K, V), torch.empty((B, K), device="cuda")
    score[:, 0], score[:, 1], score[:, 2] = -3.2e38, -3.0e38, -3.1e38
    z[:, 1] = 3e38
    z[::2, 2] = -3e38
    score[1::2, 2] = 3e38
    z[1::2, 2] = -2e38
    check_select(z.view(B * K, V), score, n)
