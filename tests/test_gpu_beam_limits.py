"""Selections at the edges of what the arithmetic holds: masks of any size, and logits and scores as large as fp32 has them."""
import math

import pytest
import torch

import test_gpu_beams as beams
from paper_2405_04304_b200 import binding
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


def best_by_sorted_sums(z, score, n, finished=None, eos=-1):
    """best_of in 64 bits with each row's exponentials added in the order of their size: rows of the same logits, wherever these stand, get the
    same sum.  Differences of neighbours of different beams are 2^-40 at least, or none: 64-bit sums are good to less than 2^-46."""
    B, K = score.shape
    z = z.double().reshape(B, K, -1).cpu()
    lse = torch.logsumexp(z.sort(2).values, 2, keepdim=True)
    l = score.double().cpu()[:, :, None] + (z - lse)
    if finished is not None:
        for b, k in finished.cpu().nonzero().tolist():
            l[b, k] = -math.inf
            l[b, k, eos] = float(score[b, k])
    V = z.shape[2]
    flat = l.reshape(B, K * V)
    at = torch.argsort(flat, dim=1, descending=True, stable=True)[:, :n + 1]
    s = flat.gather(1, at)
    gap = (s[:, :-1] - s[:, 1:])[(at[:, :-1] // V != at[:, 1:] // V)]
    assert (gap[gap != 0] > 2.0 ** -40).all()
    return s[:, :n], at[:, :n] // V, at[:, :n] % V


def check_near(z, score, n, want, finished=None, eos=-1):
    B, K = score.shape
    V = z.shape[-1]
    ctx = beams.context(V, batch=B, rows=B * K)
    s, p, t = torch.full((B, n), 7.0, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda")
    ctx.beam_select(z.view(B * K, V), score, s, p, t, finished=finished, eos=eos)
    assert ctx.device_status() == 0
    assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])
    assert ((s.cpu().double() - want[0]).abs() <= beams.score_tol(want[0])).all()


def near_scores(z, B, K):
    """Scores with which the beams' best continuations are equal but for the rounding of the scores, 2^-23 at most."""
    z = z.double().view(B, K, -1)
    best = (z.amax(2) - torch.logsumexp(z, 2))
    return (-3.0 - best).float()


@pytest.mark.parametrize("z_type", [F32, BF16, F16])
@pytest.mark.parametrize("B,K,n,V", [(8, 2, 1, 500), (8, 4, 4, 5000), (40, 4, 8, 2500), (4, 16, 16, 9001), (2, 40, 30, 700), (3, 64, 128, 2050), (1, 3, 5, 151936)])
def test_select_beams_nearer_than_fp32_sums(z_type, B, K, n, V):
    g = gen(B * 7 + K + V)
    z = (randn(g, B * K, V) * 1.5).to(z_type)
    score = near_scores(z, B, K)
    check_near(z, score, n, best_by_sorted_sums(z, score, n))


@pytest.mark.parametrize("B", [6, 40])
def test_select_ended_beams_next_to_others(B):
    """An ended beam's score is exact; a living one's continuation comes as near to it as fp32 scores allow."""
    g = gen(B)
    K, V, n = 4, 3000, 4
    z = randn(g, B * K, V) * 1.5
    score, fin = near_scores(z, B, K), torch.zeros((B, K), dtype=beams.U8, device="cuda")
    fin[:, 1] = 1
    # (scores one by one: of the same logits, the first of many near ones that is not a tie)
    score[:, 1] = (score[:, 0].double() + z.double().view(B, K, V)[:, 0].amax(1) - torch.logsumexp(z.double().view(B, K, V)[:, 0], 1)).float()
    check_near(z, score, n, best_by_sorted_sums(z, score, n, fin, 7), fin, 7)


def permuted(g, B, K, V, values):
    """K rows of the same logits, each in an order of its own."""
    z = torch.empty((B, K, V))
    for b in range(B):
        for k in range(K):
            z[b, k] = values[b][torch.randperm(V, generator=g)]
    return z.cuda()


@pytest.mark.parametrize("z_type", [F32, BF16])
@pytest.mark.parametrize("B,K,n,V", [(4, 4, 4, 5000), (40, 3, 6, 1500), (2, 16, 20, 3001), (1, 50, 100, 700)])
def test_select_equal_beams_with_their_logits_in_another_order(z_type, B, K, n, V):
    """Equal continuations of different beams: the lower beam, in whatever order its logits were added."""
    g = gen(V + K)
    z = permuted(g, B, K, V, [torch.randn(V, generator=g) * 1.5 for _ in range(B)]).to(z_type).view(B * K, V)
    score = torch.full((B, K), -2.5, device="cuda")
    check_near(z, score, n, best_by_sorted_sums(z, score, n))


@pytest.mark.parametrize("B", [2, 40])
@pytest.mark.parametrize("K,n,V,values", [(3, 100, 6000, 3), (3, 4, 6000, 3), (2, 128, 30000, 40), (4, 20, 70000, 2), (1, 30, 30000, 2), (40, 128, 1500, 2)])
def test_select_equal_beams_full_of_ties(K, n, V, values, B):
    """The same with few values: more pieces and more logits at the cut than the lists hold."""
    if B * K * V > 9_000_000:
        B = max(1, 9_000_000 // (K * V))
    g = gen(V + K + values)
    z = permuted(g, B, K, V, [torch.randint(0, values, (V,), generator=g).float() for _ in range(B)]).view(B * K, V)
    score = torch.full((B, K), -1.5, device="cuda")
    score[:, K // 2:] -= 2.0 ** -20
    check_near(z, score, n, best_by_sorted_sums(z, score, n))


def test_select_equal_logits_before_a_better_beam():
    """The n-th best and what comes behind it are equal continuations of one beam; a third, of another beam, may be better than both."""
    g = gen(77)
    B, V = 40, 2000
    z = randn(g, 2 * B, V)
    top = z.amax(1)
    z[::2, 1000] = z[::2, 10] = z[::2, 500] = top[::2] + 1.0
    score = near_scores(z, B, 2)
    for n in (1, 2):
        check_near(z, score, n, best_by_sorted_sums(z, score, n))


@pytest.mark.parametrize("V,d,B,K,n", [(5000, 256, 3, 4, 8), (700, 64, 2, 33, 20), (9001, 512, 40, 4, 4)])
def test_step_beams_nearer_than_fp32_sums(V, d, B, K, n):
    g = gen(V)
    Wq, ws = head(V, d, g)
    ws *= 55.0 / math.sqrt(d)
    H = randn(g, B * K, d).bfloat16()
    H[1] = H[0]
    z = logits_of(Wq, ws, H)
    score = near_scores(z, B, K)
    want = best_by_sorted_sums(z, score, n)
    s, p, t = torch.zeros((B, n), device="cuda"), torch.zeros((B, n), dtype=I32, device="cuda"), torch.zeros((B, n), dtype=I32, device="cuda")
    ctx = beams.context(V, d, batch=B, rows=B * K)
    ctx.beam_step_int8(Wq, ws, H, score, s, p, t, torch.empty((B * K, V), device="cuda"))
    assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])
    assert ((s.cpu().double() - want[0]).abs() <= beams.score_tol(want[0])).all()


# ------------------------------------------------------------------------------------------------ large vocabularies
def test_select_largest_vocabulary_and_one_beyond_it():
    V, K, n = 1 << 28, 34, 5
    z = torch.empty((K, V), dtype=F16, device="cuda").uniform_(-4.0, 0.0)
    at = [(33, V - 1), (0, 0), (32, 1 << 27), (33, 12345), (5, (1 << 28) - 4097)]
    for i, (k, v) in enumerate(at):
        z[k, v] = 60.0 - i
    score = torch.linspace(-1.0, -2.0, K, device="cuda")[None].contiguous()
    lse = torch.stack([torch.logsumexp(row.double(), 0) for row in z])
    l = [float(score[0, k].double() + (z[k, v].double() - lse[k])) for k, v in at]
    order = sorted(range(n), key=lambda i: -l[i])
    assert all(l[a] - l[b] > 1e-3 for a, b in zip(order, order[1:]))
    ctx = beams.context(V, d=8, batch=1, rows=K)
    s, p, t = lists_of(ctx, z, score, n)
    assert list(zip(p[0].tolist(), t[0].tolist())) == [at[i] for i in order]
    assert all(abs(float(s[0, j]) - l[i]) < 2.0 ** -20 * V / 4096 for j, i in enumerate(order))
    ctx.close()
    more = beams.context(V + 1, d=8, batch=1, rows=1)
    vp, UNS = lambda t: t.data_ptr(), binding.ERR_UNSUPPORTED_SHAPE
    s, p = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    assert more._lib.disco_beam_select(more._h, vp(z), 2, V + 1, 1, 1, vp(s), None, -1, 1, vp(s), vp(p), vp(p), None, None) == UNS
    assert more.launch_count() == 0
    more.close()
