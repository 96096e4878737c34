"""The 8-bit LM head and beam search on the GPU against plain implementations in 64 bits.

Integers (quantised rows, parents, tokens, moved states) have to be equal.  Logits of the 8-bit head see three roundings to fp32 in a
stated order, so they are equal bit for bit to the same roundings of the exact sums.  Scores: see SCORE_TOL.
"""
import math

import pytest
import torch

from paper_2405_04304_b200 import binding

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
I32, U8 = torch.int32, torch.uint8

# How far the logarithm of a row's sum of exponentials may be off, which is how far the sum may be off relatively.  A term 2^-t comes from an
# exponential good to 2^-22, of a t rounded to fp32 and formed with a rounded log2 e: weighted with the term itself, t 2^-t <= 0.53, below
# 2^-21.7 in all.  Ten additions in fp32 bring the terms of a warp together (2^-20.7), a factor makes good what the largest logit's product
# lost (2^-23); the sums of a lane's chunks, up to eight of them, meet with weights that are such terms again (2^-21.7 + 2^-21), and so do
# those of a row's warps, in 64 bits (2^-21.7): 2^-18.9.  Rows that are dealt out in several rounds repeat a weight or two.
LSE_TOL = 2.0 ** -18


def score_tol(score):
    """LSE_TOL, and the rounding of the score to fp32: half a last place."""
    return LSE_TOL + score.abs() * 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g).cuda()


def rand(g, *shape):
    return torch.rand(shape, generator=g).cuda()


def randint(g, lo, hi, shape, dtype):
    return torch.randint(lo, hi, shape, generator=g).to(dtype).cuda()


def context(V, d=64, batch=1, rows=64):
    return binding.Context(V, d, d, max_batch=batch, max_rows=rows)


# ------------------------------------------------------------------------------------------------ rows in 8 bits
def quantised(x):
    """By the definition, in 64 bits (127 x is exact there)."""
    x = x.double()
    top = x.abs().amax(1, keepdim=True)
    ok = torch.isfinite(x).all(1, keepdim=True)
    q = torch.where(ok & (top > 0), torch.round(127.0 * x / top), 0.0)
    # (on the GPU torch divides by a number by multiplying with its rounded reciprocal; by a tensor it divides)
    scale = torch.where(ok[:, 0], top[:, 0].float() / torch.full_like(top[:, 0], 127.0, dtype=F32), math.nan)
    return q.nan_to_num(0.0).to(torch.int8), scale


def check_quantised(ctx, x):
    rows, d = x.shape
    Q = torch.full((rows, binding.int8_pitch(d) + 16), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -7.0, device="cuda")
    ctx.quantize_rows(x, Q, s)
    q, scale = quantised(x)
    assert torch.equal(Q[:, :d], q)
    assert torch.equal(s, scale) or torch.equal(s.nan_to_num(-1.0), scale.nan_to_num(-1.0))
    end = binding.int8_pitch(d)
    assert (Q[:, d:end] == 0).all() and (Q[:, end:] == 77).all()
    return Q, s


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,d", [(1, 8), (3, 24), (5, 136), (7, 1000), (2, 1024), (4, 1032), (33, 2048), (2, 6144), (3, 6152), (1, 16384), (2, 3000), (3, 4096), (2, 4104), (3, 8192), (2, 8200),
                                    (2047, 136), (2049, 136), (2051, 1000), (3001, 1024), (2050, 1032), (2049, 2048), (2100, 2056), (2048, 6152)])
def test_quantised_rows(dtype, rows, d):
    ctx = context(64)
    g = gen(rows * 100 + d)
    check_quantised(ctx, randn(g, rows, d).to(dtype))
    wide = randn(g, rows, d + 24).to(dtype)                       # rows that lie apart
    check_quantised(ctx, wide[:, 8:8 + d])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantised_rows_on_the_border_between_two_integers(dtype):
    ctx = context(64)
    # 127 x / 254 = x / 2: every odd x is a tie; then the same with neighbours of ties, and with other scales
    x = torch.arange(-254, 255, device="cuda").float()
    x = torch.cat([x, torch.zeros(3, device="cuda")])[None].repeat(4, 1)
    eps = torch.finfo(dtype).eps
    x[1, :509] *= 1 + eps * (x[1, :509].abs() < 254)
    x[2, :509] *= 1 - eps * (x[2, :509].abs() < 254)
    x[3] *= 3.0
    y = (x / 64).to(dtype)
    check_quantised(ctx, y)
    assert int(quantised(y)[0][0, 1]) == -126 and int(quantised(y)[0][0, 3]) == -126      # -253 / 2 and -251 / 2: ties to even


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantised_rows_of_zeros_of_extremes_and_of_what_is_not_finite(dtype):
    ctx = context(64)
    info = torch.finfo(dtype)
    x = randn(gen(1), 9, 40).to(dtype)
    x[0] = 0
    x[1, 3] = math.nan
    x[2, 5] = math.inf
    x[3, 7] = -math.inf
    x[4] = (randn(gen(2), 40) * info.max / 8).clamp(-info.max, info.max).to(dtype)
    x[4, 11] = info.max
    x[5] = (randn(gen(3), 40) * info.tiny).to(dtype)
    x[6] = 0
    x[6, 39] = info.smallest_normal * info.eps                  # the smallest number there is
    x[7] = 0
    x[7, 0] = -info.max
    x[8, 1:] = 0
    Q, s = check_quantised(ctx, x)
    assert s[0] == 0 and torch.isnan(s[1:4]).all() and (Q[:4, :40] == 0).all()


def test_quantised_head_is_usable_by_the_next_call():
    V, d, R = 3000, 256, 3
    ctx = context(V, d, rows=R)
    g = gen(5)
    for _ in range(20):
        W, H = randn(g, V, d).bfloat16(), randn(g, R, d).bfloat16()
        Wq, ws, y = torch.zeros((V, d), dtype=torch.int8, device="cuda"), torch.zeros(V, device="cuda"), torch.zeros((R, V), device="cuda")
        ctx.quantize_rows(W, Wq, ws)
        ctx.project_int8(Wq, ws, H, y)
        assert torch.equal(y, logits_of(*quantised(W), H))


# ------------------------------------------------------------------------------------------------ the product
def logits_of(Wq, ws, H):
    """Exact sums, then the three roundings of the definition."""
    q, s = quantised(H)
    acc = q.double() @ Wq[:, :H.shape[1]].double().T             # integers below 2^53: exact
    return acc.float() * s[:, None] * ws[None, :]


def head(V, d, g, extra=0):
    Wq = randint(g, -127, 128, (V, binding.int8_pitch(d) + extra), torch.int8)   # noise behind column d
    return Wq, rand(g, V) * 1e-3


def check_project(V, d, R, h_type=BF16, y_type=F32, extra=0, pad_h=0, pad_y=0, ctx=None):
    ctx = ctx or context(V, d, rows=R)
    g = gen(V + d * 3 + R * 7)
    Wq, ws = head(V, d, g, extra)
    H = randn(g, R, d + pad_h).to(h_type)[:, :d]
    y = torch.full((R, V + pad_y), -7.0, dtype=y_type, device="cuda")
    ctx.project_int8(Wq, ws, H, y[:, :V])
    assert ctx.device_status() == 0
    assert torch.equal(y[:, :V], logits_of(Wq, ws, H).to(y_type))
    assert (y[:, V:] == -7.0).all()


@pytest.mark.parametrize("R", [1, 2, 8, 15, 16, 17, 31, 32, 33, 64, 100, 127, 128, 129, 144, 200, 255, 256, 257, 272, 300, 513, 704, 1000])
def test_project_rows(R):
    check_project(5000, 256, R)


@pytest.mark.parametrize("V,d,R", [(5000, 2048, 257), (5000, 2104, 577), (9001, 2048, 545), (18001, 2048, 704), (3001, 2504, 961), (18001, 136, 577), (5000, 136, 785)])
def test_project_with_a_last_tile_of_fewer_rows(V, d, R):
    check_project(V, d, R)


@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 127, 128, 129, 256, 257, 1000, 4001, 18944, 18945, 37888, 37889, 40011])
@pytest.mark.parametrize("R", [3, 130])
def test_project_vocabularies(V, R):
    check_project(V, 136, R)


@pytest.mark.parametrize("d", [8, 16, 24, 120, 128, 136, 248, 256, 768, 1000, 2048, 2504, 5120, 6144, 16384])
def test_project_widths(d):
    check_project(3001, d, 11)


@pytest.mark.parametrize("h_type", [BF16, F16, F32])
@pytest.mark.parametrize("y_type", [BF16, F16, F32])
def test_project_types_and_strides(h_type, y_type):
    check_project(1003, 200, 21, h_type, y_type, extra=32, pad_h=16, pad_y=5)
    check_project(1003, 200, 150, h_type, y_type, pad_y=1)


def test_project_many_items_to_a_cta():
    check_project(32000, 512, 704, BF16, BF16)
    check_project(40011, 768, 390)


def test_project_large_heads_and_many_rows():
    check_project(151936, 64, 5)
    check_project(1_000_003, 8, 2)
    check_project(3000, 264, 4100)
    check_project(200, 16384, 700, BF16, F16)


def test_project_lowest_integers():
    """-128 is no rounded number, but a head may hold it."""
    V, d, R = 1000, 776, 20
    ctx = context(V, d, rows=R)
    Wq, ws = head(V, d, gen(9))
    Wq[::3, ::2] = -128
    H, y = randn(gen(10), R, d).half(), torch.zeros((R, V), device="cuda")
    ctx.project_int8(Wq, ws, H, y)
    assert torch.equal(y, logits_of(Wq, ws, H))


def test_project_largest_sums():
    V, d, R = 300, 16384, 4
    ctx = context(V, d, rows=R)
    Wq = torch.full((V, d), 127, dtype=torch.int8, device="cuda")
    Wq[1::2] = -127
    Wq[2::3, ::2] = -127
    ws = torch.linspace(0.5, 1.5, V, device="cuda")
    H = torch.ones((R, d), dtype=BF16, device="cuda") * torch.tensor([[1.0], [-2.0], [0.25], [3.0]], dtype=BF16, device="cuda")
    y = torch.zeros((R, V), device="cuda")
    ctx.project_int8(Wq, ws, H, y)
    assert torch.equal(y, logits_of(Wq, ws, H))
    assert float(y[0, 0]) == float(torch.tensor(127.0 * 127 * d) * (torch.tensor(1.0) / torch.tensor(127.0)) * 0.5)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,d", [(9, 64), (40, 64), (16, 1000)])
def test_project_rows_of_any_size(R, d, dtype):
    """Zeros, the smallest and the largest numbers, borders between integers, what is not finite; rows rounded before and in the kernel."""
    V = 500
    ctx = context(V, d, rows=R)
    Wq, ws = head(V, d, gen(1))
    info = torch.finfo(dtype)
    H = randn(gen(2), R, d).to(dtype)
    H[3, 5], H[7, 0], H[8, 63] = math.nan, math.inf, -math.inf
    H[0] = 0
    H[1] = (randn(gen(3), d) * info.tiny).to(dtype)
    H[2] = 0
    H[2, 7] = -info.smallest_normal * info.eps
    H[4, 1] = info.max
    H[5] = torch.arange(d, device="cuda").to(dtype) % 254
    H[5, 0] = 254                                  # 127 x / 254: every odd x is a tie
    y = torch.zeros((R, V), device="cuda")
    ctx.project_int8(Wq, ws, H, y)
    want = logits_of(Wq, ws, H)
    bad = [3, 7, 8]
    assert torch.isnan(y[bad]).all() and (y[0] == 0).all()
    keep = [r for r in range(R) if r not in bad]
    # (sums times a scale of 2.7e36 pass what fp32 holds: infinities by the definition's order of roundings, equal ones)
    assert not torch.isnan(want[keep]).any() and torch.equal(y[keep], want[keep])


# ------------------------------------------------------------------------------------------------ selection
def best_of(z, score, n, finished=None, eos=-1):
    """All continuations of each sequence by score, then by place: (score, parent, token, finished) in 64 bits, from the definition."""
    B, K = score.shape
    z = z.double().reshape(B, K, -1).cpu()
    score = score.double().cpu()
    V = z.shape[2]
    out_s, out_p = torch.full((B, n), -math.inf, dtype=torch.float64), torch.full((B, n), -1)
    out_t, out_f = torch.full((B, n), -1), torch.zeros((B, n), dtype=U8)
    gap = math.inf     # smallest difference between neighbours of different beams, down to the first that is left out
    for b in range(B):
        l = torch.full((K, V), -math.inf, dtype=torch.float64)
        for k in range(K):
            if not bool(torch.isfinite(score[b, k])):
                continue
            if finished is not None and bool(finished[b, k]):
                l[k, eos] = score[b, k]
                continue
            row = z[b, k]
            if bool(torch.isnan(row).any()) or bool((row == math.inf).any()) or bool((row == -math.inf).all()):
                continue
            l[k] = score[b, k] + (row - torch.logsumexp(row, 0))
        flat = l.reshape(-1)
        order = torch.argsort(flat, descending=True, stable=True)
        order = order[flat[order] > -math.inf][:n + 1]
        for i in range(1, order.numel()):
            if order[i] // V != order[i - 1] // V and flat[order[i]] != flat[order[i - 1]]:
                gap = min(gap, float(flat[order[i - 1]] - flat[order[i]]))
        order = order[:n]
        m = order.numel()
        out_s[b, :m], out_p[b, :m], out_t[b, :m] = flat[order], order // V, order % V
        for j in range(m):
            out_f[b, j] = int(int(out_t[b, j]) == eos or (finished is not None and bool(finished[b, int(out_p[b, j])])))
    return out_s, out_p, out_t, out_f, gap


def check_select(z, score, n, finished=None, eos=-1, ctx=None, in_place=False):
    B, K = score.shape
    V = z.shape[-1]
    ctx = ctx or context(V, batch=B, rows=B * K)
    want_s, want_p, want_t, want_f, gap = best_of(z, score, n, finished, eos)
    # (no two beams' candidates nearer than what rounding may turn round: a matter of the inputs, settled before the GPU is asked)
    assert gap > 4 * LSE_TOL
    s = score.clone() if in_place else torch.full((B, n), 7.0, device="cuda")
    f = finished.clone() if in_place else torch.full((B, n), 7, dtype=U8, device="cuda")
    p, t = torch.full((B, n), -7, dtype=I32, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda")
    ctx.beam_select(z, s if in_place else score, s, p, t, finished=f if in_place else finished, eos=eos, finished_out=f)
    assert ctx.device_status() == 0
    assert torch.equal(p.cpu().long(), want_p) and torch.equal(t.cpu().long(), want_t)
    assert torch.equal(f.cpu(), want_f)
    got = s.cpu().double()
    assert torch.equal(got == -math.inf, want_s == -math.inf)
    ok = want_s > -math.inf
    assert ((got - want_s).abs()[ok] <= score_tol(want_s)[ok]).all()


def beam_scores(g, B, K):
    return -3.0 - torch.cumsum(rand(g, B, K) * 2.0, 1)


@pytest.mark.parametrize("z_type", [F32, BF16, F16])
@pytest.mark.parametrize("B,K,n,V", [(1, 1, 1, 1), (1, 1, 5, 3), (2, 3, 3, 31), (1, 4, 4, 128), (3, 4, 8, 129), (1, 8, 8, 1023), (2, 5, 10, 1025),
                                     (7, 5, 5, 4001), (1, 4, 4, 32000), (3, 16, 32, 5003), (2, 64, 64, 1000), (2, 64, 128, 300), (1, 2, 128, 40),
                                     (1, 1, 128, 20011), (5, 1, 1, 777)])
def test_select(z_type, B, K, n, V):
    g = gen(B * 1000 + K * 100 + n + V)
    z = (randn(g, B * K, V) * 2.0).to(z_type)
    check_select(z, beam_scores(g, B, K), n)


@pytest.mark.parametrize("V", list(range(1, 40)) + [1151, 1152, 1153])
def test_select_every_small_vocabulary(V):
    g = gen(V)
    check_select(randn(g, 6, V), beam_scores(g, 2, 3), 4)


def test_select_with_ended_and_dead_beams():
    g = gen(3)
    B, K, V = 6, 5, 3001
    z, score = randn(g, B * K, V), beam_scores(g, B, K)
    fin = torch.zeros((B, K), dtype=U8, device="cuda")
    score[0, 1:] = -math.inf                       # the first token
    score[1] = -math.inf                           # nothing left
    fin[2] = 1                                     # all ended
    fin[3, 0], fin[3, 3] = 1, 9
    score[4, 2], score[4, 3] = math.nan, math.inf
    fin[4, 1], score[4, 1] = 1, -math.inf          # ended and dead
    z[2 * K:3 * K] = math.nan                      # logits of beams that do not expand are not looked at
    z[1 * K:2 * K] = math.nan
    z[0 * K + 1:1 * K] = math.inf
    for n in (1, 5, 10):
        check_select(z, score, n, fin, eos=2)
        check_select(z, score, n, fin, eos=V - 1)
    check_select(z, score, 5, fin, eos=0, in_place=True)


def test_select_ends_with_the_token_without_flags():
    g = gen(4)
    z = randn(g, 8, 50)
    z[:, 7] += 9.0
    check_select(z, beam_scores(g, 2, 4), 4, None, eos=7)


@pytest.mark.parametrize("z_type", [F32, BF16, F16])
def test_select_masked_logits(z_type):
    g = gen(6)
    B, K, V = 4, 3, 2500
    z = randn(g, B * K, V).to(z_type)
    low = torch.finfo(z_type).min
    z[0, :] = -math.inf                            # a row without a token
    z[1, 5:] = -math.inf                           # few tokens
    z[3, :2499] = -math.inf                        # one token, the last
    z[4, :] = low                                  # the type's lowest value everywhere
    z[5, 100:] = low
    z[6, 17] = math.nan
    z[7, 2000] = math.inf
    z[9, ::2] = -math.inf
    z[10, 1024:1152] = -math.inf                   # a chunk without a token
    score = beam_scores(g, B, K)
    for n in (3, 12):
        check_select(z, score, n)


def test_select_equal_logits():
    """Rows full of equal logits, beams that are equal: by place alone."""
    g = gen(8)
    for V in (40, 700, 5000):
        for K, n in ((1, 100), (4, 9), (3, 128)):
            check_select(torch.zeros((2 * K, V), device="cuda"), torch.full((2, K), -1.0, device="cuda"), n)
            z = randint(g, -3, 2, (2 * K, V), F32)
            z = z[:1].repeat(2 * K, 1).contiguous()      # the same row for all beams: equal scores
            check_select(z, torch.full((2, K), -1.0, device="cuda"), n)
    z = torch.zeros((64, 300), device="cuda")
    check_select(z, torch.zeros((1, 64), device="cuda"), 128)     # more candidates than are ranked at once, all equal
    z[:, 5] = -0.0
    check_select(z, torch.zeros((1, 64), device="cuda"), 128)


def test_select_more_candidates_than_are_ranked_at_once():
    g = gen(9)
    check_select(randn(g, 64, 2000) * 3.0, -torch.arange(64, device="cuda")[None] * 0.37, 128)


def test_select_rows_that_lie_apart_at_any_alignment():
    g = gen(10)
    for z_type in (F32, BF16):
        wide = randn(g, 8, 1301).to(z_type)
        for at in (0, 1, 3):
            check_select(wide[:, at:at + 1290], beam_scores(g, 2, 4), 4)


def test_select_equal_beams_at_different_alignments_are_equal():
    """Sums do not depend on where a row lies."""
    g = gen(11)
    row = randn(g, 1, 5003)
    check_select(row.repeat(4, 1).contiguous(), torch.full((1, 4), -2.0, device="cuda"), 9)


def test_select_large_rows():
    g = gen(12)
    V = 300_001        # more chunks than have their keys in shared memory are in the next one
    check_select(randn(g, 2, V), beam_scores(g, 1, 2), 4)
    V = 1_100_000
    check_select(randn(g, 1, V), beam_scores(g, 1, 1), 3)


@pytest.mark.parametrize("K,n,V", [(7, 7, 3000), (8, 8, 9000), (9, 12, 2000), (16, 24, 30000), (17, 17, 2500), (31, 40, 1200), (32, 32, 5000), (33, 33, 900), (40, 80, 4100),
                                   (63, 20, 2050), (64, 10, 20011), (48, 100, 18500)])
def test_select_beams_dealt_to_warps(K, n, V):
    """One, two and more warps to a beam, two beams to a warp, several chunks to a piece."""
    g = gen(K * 7 + n)
    z, score = randn(g, 2 * K, V) * 1.5, beam_scores(g, 2, K) * 0.2
    score[1, K // 2:] = -math.inf
    check_select(z, score, n)


def test_select_scores_of_any_size():
    """Scores that leave nothing of the logits' differences (equal, then: by place), and logits of any size."""
    g = gen(17)
    z = randn(g, 12, 700)
    score = torch.tensor([[-1e30, -1e30, -3e38], [1e30, 1e30, 0.0], [3e38, -3e38, -3e38], [0.0, -0.0, -1e-40]], device="cuda")
    z[3] *= 1e30
    z[8] = 3e38
    z[8, 100:] = -3e38
    check_select(z, score, 9)


def test_select_logits_on_a_coarse_grid():
    """bf16 logits with few values: many pieces hold the same best one."""
    g = gen(18)
    z = (randn(g, 20, 30000) * 2.0).round().bfloat16()
    check_select(z, beam_scores(g, 4, 5), 10)
    check_select(z[:4], beam_scores(g, 1, 4), 128)


def test_select_twice_on_one_context_and_captured():
    g = gen(13)
    B, K, V = 3, 4, 2000
    ctx = context(V, batch=B, rows=B * K)
    z, score = randn(g, B * K, V), beam_scores(g, B, K)
    s, p, t = torch.zeros((B, K), device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda")
    ctx.beam_select(z, score, s, p, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.beam_select(z, score, s, p, t)
    for seed in (1, 2, 3):
        z.copy_(randn(gen(seed), B * K, V))
        graph.replay()
        want = best_of(z, score, K)
        assert want[4] > 4 * LSE_TOL
        assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])


# ------------------------------------------------------------------------------------------------ both at once
def check_step(V, d, B, K, n, h_type=BF16, finished=None, first=False, seed=0):
    ctx = context(V, d, batch=B, rows=B * K)
    g = gen(V + d + B * 10 + K + seed)
    Wq, ws = head(V, d, g)
    ws *= 55.0 / math.sqrt(d)      # logits of a spread of about 2
    H = randn(g, B * K, d).to(h_type)
    score = beam_scores(g, B, K)
    if first:
        score[:, 1:] = -math.inf
    z = logits_of(Wq, ws, H)
    want_s, want_p, want_t, want_f, gap = best_of(z, score, n, finished, min(2, V - 1))
    assert gap > 4 * LSE_TOL
    s, f = torch.full((B, n), 7.0, device="cuda"), torch.full((B, n), 7, dtype=U8, device="cuda")
    p, t = torch.full((B, n), -7, dtype=I32, device="cuda"), torch.full((B, n), -7, dtype=I32, device="cuda")
    work = torch.empty((B * K, V), device="cuda")
    ctx.beam_step_int8(Wq, ws, H, score, s, p, t, work, finished=finished, eos=min(2, V - 1), finished_out=f)
    assert ctx.device_status() == 0
    assert torch.equal(p.cpu().long(), want_p) and torch.equal(t.cpu().long(), want_t) and torch.equal(f.cpu(), want_f)
    ok = want_s > -math.inf
    assert ((s.cpu().double() - want_s).abs()[ok] <= score_tol(want_s)[ok]).all()


@pytest.mark.parametrize("V,d,B,K,n", [(1, 8, 1, 1, 1), (31, 16, 1, 2, 3), (33, 24, 2, 2, 2), (257, 64, 3, 5, 5), (4001, 136, 2, 4, 8), (5000, 1000, 16, 8, 8),
                                       (32000, 768, 1, 4, 4), (9003, 256, 70, 4, 4), (3001, 264, 9, 64, 64), (40011, 128, 5, 5, 5)])
def test_step(V, d, B, K, n):
    check_step(V, d, B, K, n)


def test_step_first_token_types_and_ended_beams():
    check_step(3000, 200, 4, 5, 5, first=True)
    check_step(3000, 200, 4, 5, 5, h_type=F16)
    fin = torch.zeros((4, 5), dtype=U8, device="cuda")
    fin[0, 1] = fin[2] = 1
    check_step(3000, 200, 4, 5, 10, h_type=F32, finished=fin)


def test_step_with_hidden_states_that_are_not_numbers():
    V, d, B, K = 2000, 64, 2, 3
    ctx = context(V, d, batch=B, rows=B * K)
    g = gen(21)
    Wq, ws = head(V, d, g)
    ws *= 7.0                      # logits of a spread of about 2
    H, score = randn(g, B * K, d).bfloat16(), beam_scores(g, B, K)
    H[1, 3], H[3:] = math.nan, math.inf
    s, p, t = torch.zeros((B, K), device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda")
    ctx.beam_step_int8(Wq, ws, H, score, s, p, t, torch.empty((B * K, V), device="cuda"))
    want = best_of(logits_of(Wq, ws, H), score, K)
    assert want[4] > 4 * LSE_TOL
    assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])
    assert (p[1] == -1).all() and (t[1] == -1).all() and not (p[0] == 1).any()


def test_step_with_equal_beams_and_one_that_is_not_a_number():
    """Beams that are equal stay equal, whatever their neighbours are: the lower one first."""
    V, d, K = 3000, 128, 40
    ctx = context(V, d, batch=1, rows=K)
    g = gen(23)
    Wq, ws = head(V, d, g)
    ws *= 5.0
    H, score = randn(g, K, d).bfloat16(), beam_scores(g, 1, K)
    H[17], H[39] = H[0], H[0]
    score[0, 17] = score[0, 39] = score[0, 0]
    H[1, 3], H[35, 0] = math.nan, math.inf
    n = 24
    s, p, t = torch.zeros((1, n), device="cuda"), torch.zeros((1, n), dtype=I32, device="cuda"), torch.zeros((1, n), dtype=I32, device="cuda")
    ctx.beam_step_int8(Wq, ws, H, score, s, p, t, torch.empty((K, V), device="cuda"))
    want = best_of(logits_of(Wq, ws, H), score, n)
    assert want[4] > 4 * LSE_TOL
    assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])
    assert p[0, :3].tolist() == [0, 17, 39]


# ------------------------------------------------------------------------------------------------ states
def moved(src, dst, parent, lens=None, length_dim=1):
    B, n = parent.shape
    K = src.shape[0] // B
    out = dst.clone()
    for b in range(B):
        for j in range(n):
            k = int(parent[b, j])
            if not 0 <= k < K:
                continue
            if lens is None:
                out[b * n + j] = src[b * K + k]
            else:
                used = min(max(int(lens[b]), 0), src.shape[length_dim])
                at = (slice(None),) * (length_dim - 1) + (slice(0, used),)
                out[(b * n + j,) + at] = src[(b * K + k,) + at]
    return out


def states(g, rows, shape, dtype):
    if dtype.is_floating_point:
        return randn(g, rows, *shape).to(dtype)
    return randint(g, 0, 100, (rows, *shape), dtype)


@pytest.mark.parametrize("dtype,shape", [(BF16, (4, 33, 8)), (F32, (3, 17, 5)), (U8, (2, 7, 3)), (BF16, (1, 9, 3)), (I32, (300,)), (torch.int64, (5, 2)),
                                         (U8, (1,)), (torch.float64, ()), (BF16, (2, 5000, 64))])
@pytest.mark.parametrize("B,K,n", [(1, 1, 1), (2, 4, 4), (3, 5, 10), (1, 16, 16), (2, 33, 20), (1, 64, 128)])
def test_reorder(dtype, shape, B, K, n):
    ctx = context(8)
    g = gen(B + K * 3 + n)
    parent = randint(g, 0, K, (B, n), I32)
    src = [states(g, B * K, shape, dtype) for _ in range(3)]
    dst = [states(g, B * n, shape, dtype) for _ in range(3)]
    want = [moved(s, d, parent.cpu()) for s, d in zip(src, dst)]
    ctx.beam_reorder(src, dst, parent)
    assert all(torch.equal(a, b) for a, b in zip(dst, want))
    if n == K:      # in place
        want = [moved(s, s, parent.cpu()) for s in src]
        ctx.beam_reorder(src, src, parent)
        assert all(torch.equal(a, b) for a, b in zip(src, want))
    assert ctx.device_status() == 0


@pytest.mark.parametrize("K", [2, 4, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("dtype,width", [(BF16, 8), (BF16, 4), (F32, 1), (BF16, 1), (U8, 1)])
def test_reorder_in_place(K, dtype, width):
    ctx = context(8)
    g = gen(K * 10 + width)
    B, T = 3, 70
    src = states(g, B * K, (2, T, width), dtype)
    for parent in (randint(g, 0, K, (B, K), I32),
                   torch.arange(K - 1, -1, -1, device="cuda", dtype=I32).repeat(B, 1),                 # a permutation
                   torch.roll(torch.arange(K, device="cuda", dtype=I32), 1).repeat(B, 1).contiguous(),
                   torch.zeros((B, K), dtype=I32, device="cuda")):
        lens = torch.tensor([T, 0, 33], dtype=I32, device="cuda")
        for ln in (None, lens):
            want = moved(src, src, parent.cpu(), ln, 2)
            ctx.beam_reorder([src], [src], parent, lens=ln, length_dim=2)
            assert torch.equal(src, want)


@pytest.mark.parametrize("length_dim,shape", [(1, (50, 3, 8)), (2, (3, 50, 8)), (3, (2, 3, 50)), (1, (50,)), (3, (2, 3, 50, 1))])
def test_reorder_lengths(length_dim, shape):
    ctx = context(8)
    g = gen(length_dim)
    B, K, n = 5, 4, 6
    parent = randint(g, 0, K, (B, n), I32)
    lens = torch.tensor([0, 1, 49, 50, -3], dtype=I32, device="cuda")
    for ln in (lens, torch.tensor([51, 1 << 30, 7, 8, 9], dtype=I32, device="cuda")):
        for dtype in (BF16, F32, U8):
            src, dst = states(g, B * K, shape, dtype), states(g, B * n, shape, dtype)
            want = moved(src, dst, parent.cpu(), ln, length_dim)
            ctx.beam_reorder([src], [dst], parent, lens=ln, length_dim=length_dim)
            assert torch.equal(dst, want)


def test_reorder_places_without_a_parent_and_bad_parents():
    ctx = context(8)
    g = gen(3)
    src, dst = states(g, 8, (10,), F32), states(g, 8, (10,), F32)
    parent = torch.tensor([[0, -1, 3, 2], [-1, -1, -1, 1]], dtype=I32, device="cuda")
    want = moved(src, dst, parent.cpu())
    ctx.beam_reorder([src], [dst], parent)
    assert torch.equal(dst, want) and ctx.device_status() == 0
    parent = torch.tensor([[0, 4, 3, -2], [1 << 30, 2, -(1 << 31), 1]], dtype=I32, device="cuda")
    want = moved(src, dst, parent.cpu())
    ctx.beam_reorder([src], [dst], parent)
    assert torch.equal(dst, want) and ctx.device_status() == binding.ERR_INVALID_ARG


def test_reorder_many_tensors_at_any_alignment():
    ctx = context(8)
    g = gen(4)
    B, K = 2, 3
    parent = randint(g, 0, K, (B, K), I32)
    src = [states(g, B * K, (9, 4), BF16) for _ in range(130)]
    dst = [states(g, B * K, (9, 4), BF16) for _ in range(130)]
    want = [moved(s, d, parent.cpu()) for s, d in zip(src, dst)]
    ctx.beam_reorder(src, dst, parent)
    assert all(torch.equal(a, b) for a, b in zip(dst, want))
    flat = states(g, 1, (B * K * 40 + 3,), BF16)[0]
    for at in (1, 2, 3):
        s = flat[at:at + B * K * 40].view(B * K, 40)
        d = torch.zeros_like(s)
        ctx.beam_reorder([s], [d], parent)
        assert torch.equal(d, moved(s, d, parent.cpu()))


# ------------------------------------------------------------------------------------------------ as they are used together
def reference_decode(Wq, ws, E, start, B, K, eos, steps):
    """A decoder whose hidden state is the mean of its tokens' embeddings, with beams, in plain steps."""
    hist = torch.full((B * K, steps), -1, dtype=I32)
    score = torch.full((B, K), -math.inf)
    score[:, 0] = 0.0
    fin = torch.zeros((B, K), dtype=U8)
    H = start.repeat_interleave(K, 0)
    for i in range(steps):
        z = logits_of(Wq, ws, H)
        s, p, t, f, gap = best_of(z, score, K, fin, eos)
        assert gap > 64 * LSE_TOL        # (what the scores of several steps may differ by)
        rows = (torch.arange(B)[:, None] * K + p).reshape(-1)
        hist = hist[rows]
        hist[:, i] = t.reshape(-1).to(I32)
        H = ((H[rows.cuda()].float() + E[t.reshape(-1).cuda()].float()) * 0.5).bfloat16()
        score, fin = s.float(), f
    return hist, score, fin


@pytest.mark.parametrize("captured", [False, True])
def test_decoding_with_beams(captured):
    V, d, B, K, steps, eos = 3001, 136, 3, 4, 7, 11
    g = gen(31)
    W, E, start = randn(g, V, d).bfloat16() * 0.2, randn(g, V, d).bfloat16(), randn(g, B, d).bfloat16()
    W[eos] *= 1.5
    ctx = context(V, d, batch=B, rows=B * K)
    Wq, ws = torch.empty((V, binding.int8_pitch(d)), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    ctx.quantize_rows(W, Wq, ws)
    want_hist, want_score, want_fin = reference_decode(Wq, ws, E, start, B, K, eos, steps)

    hist = torch.full((B * K, steps), -1, dtype=I32, device="cuda")
    score = torch.full((B, K), -math.inf, device="cuda")
    score[:, 0] = 0.0
    fin = torch.zeros((B, K), dtype=U8, device="cuda")
    H = start.repeat_interleave(K, 0).contiguous()
    parent, token = torch.zeros((B, K), dtype=I32, device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda")
    work = torch.empty((B * K, V), device="cuda")
    length = torch.zeros(B, dtype=I32, device="cuda")
    at = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        ctx.beam_step_int8(Wq, ws, H, score, score, parent, token, work, finished=fin, eos=eos, finished_out=fin)
        ctx.beam_reorder([hist], [hist], parent, lens=length, length_dim=1)       # tokens so far
        ctx.beam_reorder([H], [H], parent)                                       # hidden states
        hist.index_copy_(1, at, token.view(-1, 1))
        H.copy_(((H.float() + E[token.view(-1).long()].float()) * 0.5).bfloat16())
        length.add_(1)
        at.add_(1)

    if captured:
        saved = [t.clone() for t in (hist, score, fin, H, length, at)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for t, s in zip((hist, score, fin, H, length, at), saved):
            t.copy_(s)
    for _ in range(steps):
        graph.replay() if captured else step()
    assert ctx.device_status() == 0
    assert torch.equal(hist.cpu(), want_hist) and torch.equal(fin.cpu(), want_fin)
    assert ((score.cpu() - want_score).abs() <= steps * score_tol(want_score)).all()


def test_beams_on_another_stream_beside_other_calls():
    """A context of its own on a stream of its own, while another stream is at work."""
    V, d, B, K = 4000, 128, 4, 4
    g = gen(41)
    Wq, ws = head(V, d, g)
    ws *= 5.0                      # logits of a spread of about 2
    H, score = randn(g, B * K, d).bfloat16(), beam_scores(g, B, K)
    want = best_of(logits_of(Wq, ws, H), score, K)
    assert want[4] > 4 * LSE_TOL
    contexts = [context(V, d, batch=B, rows=B * K) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[(torch.zeros((B, K), device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda"),
             torch.empty((B * K, V), device="cuda")) for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(10):
        for ctx, st, o in zip(contexts, streams, out):
            ctx.beam_step_int8(Wq, ws, H, score, *o[i], stream=st)
    torch.cuda.synchronize()
    for o in out:
        for s, p, t, _ in o:
            assert torch.equal(p.cpu().long(), want[1]) and torch.equal(t.cpu().long(), want[2])


def test_other_calls_of_the_same_context_keep_their_results():
    """Draft steps and beam steps on one context in turn."""
    from paper_2405_04304_b200 import inputs
    V, d, B, K = 4096, 256, 2, 4
    ctx = binding.Context(V, d, d, max_batch=B * K, max_rows=B * K, clf_hidden=16)
    W = inputs.lm_head(V, d, 1, device="cuda", std=0.05)
    H = inputs.hidden(B * K, d, 2, device="cuda")
    clf = binding.Classifier(*(t.cuda() for t in inputs.classifier_params(16, 3)))
    pos = torch.ones(B * K, dtype=I32, device="cuda")
    Wq, ws = torch.empty((V, d), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    work = torch.empty((B * K, V), device="cuda")
    score = beam_scores(gen(1), B, K)
    seen = []
    for _ in range(4):
        token, conf, halt = torch.zeros(B * K, dtype=I32, device="cuda"), torch.zeros(B * K, device="cuda"), torch.zeros(B * K, dtype=U8, device="cuda")
        s, p, t = torch.zeros((B, K), device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda"), torch.zeros((B, K), dtype=I32, device="cuda")
        ctx.draft_step(W, H, pos, pos, clf, 0.5, 5, token, conf, halt)
        ctx.quantize_rows(W, Wq, ws)
        ctx.beam_step_int8(Wq, ws, H, score, s, p, t, work)
        ctx.draft_step(W, H, pos, pos, clf, 0.5, 5, token, conf, halt)
        seen.append((token, conf, halt, s, p, t))
    want = best_of(logits_of(*quantised(W), H), score, K)
    assert ctx.device_status() == 0
    assert torch.equal(seen[0][0].cpu(), (H.float() @ W.float().T).argmax(1).to(I32).cpu())
    for got in seen:
        assert all(torch.equal(a, b) for a, b in zip(got, seen[0]))
        assert torch.equal(got[4].cpu().long(), want[1]) and torch.equal(got[5].cpu().long(), want[2])


def test_projects_on_many_streams_at_once():
    V, d, R = 9001, 512, 160
    g = gen(61)
    Wq, ws = head(V, d, g)
    H = [randn(g, R, d).bfloat16() for _ in range(6)]
    want = [logits_of(Wq, ws, h) for h in H]
    contexts, streams = [context(V, d, rows=R) for _ in H], [torch.cuda.Stream() for _ in H]
    y = [torch.zeros((R, V), device="cuda") for _ in H]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, st, h, out in zip(contexts, streams, H, y):
            c.project_int8(Wq, ws, h, out, stream=st)
    torch.cuda.synchronize()
    for c, out, w in zip(contexts, y, want):
        assert torch.equal(out, w) and c.device_status() == 0


# ------------------------------------------------------------------------------------------------ what is refused
def refused(code, call, *args, **kw):
    with pytest.raises(binding.DiscoError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_refusals():
    V, d, B, K = 100, 32, 2, 3
    ctx = context(V, d, batch=B, rows=B * K)
    z = lambda *s, dtype=F32: torch.zeros(s, dtype=dtype, device="cuda")
    INV, UNS, WS = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED_SHAPE, binding.ERR_WORKSPACE
    # rows
    refused(INV, ctx.quantize_rows, z(2, 12), z(2, 16, dtype=torch.int8), z(2))                       # width not a multiple of 8
    refused(UNS, ctx.quantize_rows, z(1, 16392), z(1, 16400, dtype=torch.int8), z(1))
    refused(INV, ctx.quantize_rows, z(2, 41)[:, 1:33], z(2, 32, dtype=torch.int8), z(2))              # alignment
    refused(INV, ctx.quantize_rows, z(2, 36)[:, :32], z(2, 40, dtype=torch.int8), z(2))               # pitch of q
    with pytest.raises(ValueError):
        ctx.quantize_rows(z(2, 32), z(2, 16, dtype=torch.int8), z(2))
    with pytest.raises(TypeError):
        ctx.quantize_rows(z(2, 32, dtype=I32), z(2, 32, dtype=torch.int8), z(2))
    # product
    Wq, ws = z(V, 32, dtype=torch.int8), z(V)
    refused(WS, ctx.project_int8, Wq, ws, z(7, 32), z(7, V))
    refused(WS, ctx.project_int8, z(V, 64, dtype=torch.int8), ws, z(2, 64), z(2, V))                  # wider than the context
    refused(INV, ctx.project_int8, z(V, 16, dtype=torch.int8), ws, z(2, 32), z(2, V))                 # head narrower than the rows
    refused(INV, ctx.project_int8, z(V * 40 + 1, dtype=torch.int8)[1:].view(V, 40), ws, z(2, 32), z(2, V))
    for bad in (dict(H=z(2, 32).cpu()), dict(y=z(2, V + 1)), dict(y=z(3, V)), dict(ws=z(V - 1)), dict(Wq=z(V + 1, 32, dtype=torch.int8)),
                dict(y=z(V, 2).T), dict(H=z(1, 32).expand(2, 32))):
        with pytest.raises((ValueError, TypeError)):
            a = dict(Wq=Wq, ws=ws, H=z(2, 32), y=z(2, V)) | bad
            ctx.project_int8(a["Wq"], a["ws"], a["H"], a["y"])
    # selection
    score, fin = z(B, K), z(B, K, dtype=U8)
    out = lambda n: (z(B, n), z(B, n, dtype=I32), z(B, n, dtype=I32))
    refused(INV, ctx.beam_select, z(B * K, V), score, *out(K), finished=fin)                          # ended beams, but no token for it
    refused(INV, ctx.beam_select, z(B * K, V), score, *out(K), eos=V)
    refused(INV, ctx.beam_select, z(B * K, V), score, *out(K), eos=-2)
    refused(UNS, ctx.beam_select, z(B * K, V), score, *out(129))
    refused(INV, ctx.beam_select, z(B * K, V), score, *out(0))
    refused(WS, ctx.beam_select, z(2 * B * K, V), z(2 * B, K), z(2 * B, K), z(2 * B, K, dtype=I32), z(2 * B, K, dtype=I32))
    refused(UNS, ctx.beam_select, z(65, V), z(1, 65), z(1, 1), z(1, 1, dtype=I32), z(1, 1, dtype=I32))
    with pytest.raises(ValueError):
        ctx.beam_select(z(B * K, V), score, z(B, 4), z(B, 4, dtype=I32), z(B, 3, dtype=I32))
    with pytest.raises(ValueError):
        ctx.beam_select(z(B * K + 1, V), score, *out(K))
    with pytest.raises(TypeError):
        ctx.beam_select(z(B * K, V, dtype=torch.float64), score, *out(K))
    lib, vp = ctx._lib, lambda t: t.data_ptr()
    flat = z(B * 8)
    assert lib.disco_beam_select(ctx._h, vp(z(B * K, V)), 0, V, B, K, vp(flat), None, -1, K + 1, vp(flat), vp(z(16, dtype=I32)), vp(z(16, dtype=I32)),
                                 None, None) == INV                                                    # in place with another shape
    assert lib.disco_beam_select(ctx._h, vp(z(B * K, V)), 3, V, B, K, vp(flat), None, -1, K, vp(z(16)), vp(z(16, dtype=I32)), vp(z(16, dtype=I32)),
                                 None, None) == INV                                                    # no such type
    with pytest.raises(ValueError):
        ctx.beam_step_int8(Wq, ws, z(B * K, 32), score, *out(K), z(B * K, V - 1))
    # states
    parent = z(B, K, dtype=I32)
    with pytest.raises(ValueError):
        ctx.beam_reorder([z(B * K, 4)], [z(B * K, 5)], parent)
    with pytest.raises(ValueError):
        ctx.beam_reorder([z(B * K, 4)], [], parent)
    with pytest.raises(ValueError):
        ctx.beam_reorder([z(4, B * K).T], [z(B * K, 4)], parent)
    with pytest.raises(ValueError):
        ctx.beam_reorder([z(B * K, 4)], [z(B * K, 4)], parent, lens=z(B + 1, dtype=I32))
    buf = z(100, 4)
    refused(INV, ctx.beam_reorder, [buf[:6]], [buf[2:8]], parent)                                      # overlap
    refused(INV, ctx.beam_reorder, [buf[:6], buf[10:16]], [buf[:6], buf[20:26]], parent)               # some in place
    refused(INV, ctx.beam_reorder, [buf[:6]], [buf[:8]], z(B, 4, dtype=I32))                           # in place, another number
    refused(UNS, ctx.beam_reorder, [z(65, 4)], [z(1, 4)], z(1, 1, dtype=I32))
    refused(INV, ctx.beam_reorder, [z(B * K, 0)], [z(B * K, 0)], parent)
    assert ctx.device_status() == 0 and ctx.launch_count() == 0


def test_offsets_beyond_32_bits():
    g = gen(77)
    far = (1 << 31) + 4096                                   # bytes, a multiple of all sizes
    buf = torch.zeros(7 << 30, dtype=U8, device="cuda")

    def apart(x, step=far):                                  # the rows of x, `step` bytes apart
        assert x.shape[0] * step <= buf.numel()
        return buf.view(x.dtype).as_strided(x.shape, (step // x.element_size(), 1)).copy_(x)

    # rows to 8 bits, to rows that lie apart too
    x = randn(g, 3, 264).to(BF16)
    q, scale = torch.zeros((3, 272), dtype=torch.int8, device="cuda"), torch.zeros(3, device="cuda")
    ctx = context(400, 264, batch=1, rows=24)
    ctx.quantize_rows(apart(x), q, scale)
    want_q, want_scale = quantised(x)
    assert torch.equal(q[:, :264].double(), want_q.double()) and torch.equal(scale, want_scale)
    q_far = buf[:3 * far].view(torch.int8).view(3, far)      # (rows in 8 bits: contiguous, as wide as they are apart)
    q_far[:, :300] = 9
    ctx.quantize_rows(x, q_far, scale)
    assert torch.equal(q_far[:, :264], q[:, :264]) and (q_far[:, 264:272] == 0).all() and (q_far[:, 272:300] == 9).all()
    # hidden rows, logits and a head that lie apart
    Wq, ws = head(400, 264, g)
    for R in (3, 20):                                        # (rounded by the product's kernel, and before it)
        H = randn(g, R, 264).to(BF16)
        want = logits_of(Wq, ws, H)
        y = torch.zeros((R, 400), device="cuda")
        step = far if R == 3 else 1 << 28
        ctx.project_int8(Wq, ws, apart(H, step), y)
        assert torch.equal(y, want)
        y_far = apart(torch.zeros_like(y), step)
        ctx.project_int8(Wq, ws, H, y_far)
        assert torch.equal(y_far, want)
        y.zero_()
        W_far = buf[:400 << 24].view(torch.int8).view(400, 1 << 24)      # 6.7 GB
        W_far[:, :Wq.shape[1]] = Wq
        ctx.project_int8(W_far, ws, H, y)
        assert torch.equal(y, want)
    # logits that lie apart; one launch, and two
    for V in (400, 20011):
        check_select(apart(randn(g, 3, V)), beam_scores(g, 1, 3), 4)
    # states
    state = buf[:2 * far].view(2, 2, far // 2)               # [beam, head, position]
    for beam in range(2):
        state[beam, 0].fill_(3 + beam)
        state[beam, 1].fill_(5 + beam)
    both = torch.tensor([[1, 0]], dtype=I32, device="cuda")
    ctx.beam_reorder([state], [state], both)
    for beam in range(2):
        assert (state[beam, 0] == 4 - beam).all() and (state[beam, 1] == 6 - beam).all()
    parent, child = buf[:far].view(1, far), buf[far:3 * far].view(2, far)
    used = (1 << 31) - 1
    parent.copy_(torch.arange(251, dtype=U8, device="cuda").repeat(far // 251 + 1)[:far])
    child.fill_(253)
    ctx.beam_reorder([parent], [child], torch.zeros((1, 2), dtype=I32, device="cuda"), lens=torch.full((1,), used, dtype=I32, device="cuda"))
    for row in child:
        assert torch.equal(row[:used], parent[0, :used]) and (row[used:] == 253).all()
    assert ctx.device_status() == 0


def test_reorder_refuses_states_that_share_memory():
    ctx = context(8)
    parent = torch.tensor([[1, 0], [1, 1]], dtype=I32, device="cuda")
    buf = torch.arange(400, device="cuda").reshape(100, 4).float()
    at = [buf[i:i + 4] for i in range(97)]
    before = buf.clone()
    INV = binding.ERR_INVALID_ARG
    refused(INV, ctx.beam_reorder, [at[0], at[0]], [at[0], at[0]], parent)                             # a state twice, in place
    refused(INV, ctx.beam_reorder, [at[0], at[20], at[3]], [at[0], at[20], at[3]], parent)             # ... or a part of it
    refused(INV, ctx.beam_reorder, [at[0], at[10]], [at[20], at[20]], parent)                          # one place for two states
    refused(INV, ctx.beam_reorder, [at[0], at[10]], [at[20], at[23]], parent)
    refused(INV, ctx.beam_reorder, [at[0], at[10]], [at[10], at[20]], parent)                          # another state's place
    refused(INV, ctx.beam_reorder, [at[0], at[10]], [at[20], at[3]], parent)
    refused(INV, ctx.beam_reorder, [at[10], at[3]], [at[20], at[0]], parent)
    refused(INV, ctx.beam_reorder, [at[0], at[10]], [at[10], at[0]], parent)                           # exchanged
    assert torch.equal(buf, before) and ctx.launch_count() == 0
    ctx.beam_reorder([at[0], at[0], at[4]], [at[8], at[12], at[16]], parent)                           # one source for two, neighbours
    ctx.beam_reorder([at[40], at[44]], [at[40], at[44]], parent)
    rows = [1, 0, 3, 3]
    assert torch.equal(buf[8:20], torch.cat([before[0:4][rows], before[0:4][rows], before[4:8][rows]]))
    assert torch.equal(buf[40:48], torch.cat([before[40:44][rows], before[44:48][rows]]))
    assert torch.equal(buf[:8], before[:8]) and torch.equal(buf[20:40], before[20:40]) and torch.equal(buf[48:], before[48:])
    assert ctx.device_status() == 0


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_another_current_device_is_refused():
    ctx = context(100)
    z = torch.zeros((2, 32), device="cuda:0")
    with torch.cuda.device(1):
        refused(binding.ERR_INVALID_ARG, ctx.quantize_rows, z, torch.zeros((2, 32), dtype=torch.int8, device="cuda:0"), torch.zeros(2, device="cuda:0"))
        with pytest.raises(ValueError):
            ctx.quantize_rows(z.to("cuda:1"), torch.zeros((2, 32), dtype=torch.int8, device="cuda:0"), torch.zeros(2, device="cuda:0"))
