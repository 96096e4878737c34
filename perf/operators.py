"""What the beam-search operators and the 8-bit LM head are measured on.

A decoder with beams runs, for every token, an LM head over all beams (here in 8-bit integers, with a scale for each
hidden row and each vocabulary row), selects the best continuations over beams and vocabulary, and moves the beams'
states (caches, token histories) to where their parents were.  project_int8, beam_select and beam_reorder are these
three; beam_step_int8 is the first two in one call.

The head shapes are those of inputs.WORKLOADS and of the cases in perf/cases.py, from one sequence to 64; draw() gives
further ones of the same ranges (vocabulary 4000 .. 49152, odd sizes included; hidden widths, multiples of 8, 256 ..
6144; 1 .. 704 hidden rows; 1 .. 64 sequences of 1 .. 16 beams; caches of 16 .. 1024 positions).
"""
import math

import torch

own = False

EOS = 2
HEAD_STD = 0.02
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # One token of one sequence on the draft head: the smallest product, made for every token.
        dict(name="project_1", kind="project", V=32000, d=768, R=1, x="bf16", y="f32"),
        # One verification of one sequence with the full look-ahead, target head.
        dict(name="project_11", kind="project", V=32000, d=5120, R=11, x="bf16", y="f32"),
        # Tokens added to a tokeniser, an odd number of rows, half precision in and out.
        dict(name="project_23_odd", kind="project", V=40011, d=1000, R=23, x="f16", y="f16"),
        # Verification of a serving batch: 64 sequences, 11 rows each.
        dict(name="project_704", kind="project", V=32000, d=5120, R=704, x="bf16", y="bf16"),
        # One sequence, four beams: the smallest selection.
        dict(name="select_4", kind="select", V=32000, B=1, K=4, n=4, z="f32", ended=0, first=False),
        # Twice as many kept as there are beams, some of them ended, an odd vocabulary, bf16 logits (full of ties).
        dict(name="select_20x5_odd", kind="select", V=40011, B=20, K=5, n=10, z="bf16", ended=1, first=False),
        # A serving batch, eight beams.
        dict(name="select_64x8", kind="select", V=49152, B=64, K=8, n=8, z="f32", ended=0, first=False),
        # Token histories of one sequence: the smallest move of states.
        dict(name="reorder_tokens", kind="reorder", B=1, K=4, n=4, tensors=1, heads=1, T=64, D=1, t="i32", ragged=False),
        # Caches of a batch: keys and values of 12 layers, sequences of different lengths.
        dict(name="reorder_caches", kind="reorder", B=16, K=4, n=4, tensors=24, heads=12, T=512, D=64, t="bf16", ragged=True),
        # A token of one sequence with four beams on the draft head.
        dict(name="step_1x4", kind="step", V=32000, d=768, B=1, K=4, n=4, ended=0, first=False),
        # The first token of a batch (one live beam a sequence), odd vocabulary.
        dict(name="step_12x5_first", kind="step", V=40011, d=2048, B=12, K=5, n=5, ended=0, first=True),
        # A serving batch on the target head.
        dict(name="step_64x4", kind="step", V=32000, d=5120, B=64, K=4, n=4, ended=1, first=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["project", "project", "select", "reorder", "step", "step"])
    V, d = log_int(4000, 49152), 8 * log_int(32, 768)
    K = rng.randint(1, 16)
    n = rng.choice([K, 2 * K, rng.randint(1, 2 * K)])
    if kind == "project":
        most = 704 * 32000 * 5120 // (V * d)      # no more work than the largest listed case
        return dict(kind=kind, V=V, d=d, R=log_int(1, min(704, most)), x=rng.choice(["bf16", "f16", "f32"]),
                    y=rng.choice(["f32", "bf16", "f16"]))
    B = log_int(1, max(1, 64 * 8 // K) if K > 8 else 64)
    if kind == "reorder":
        T, heads, D = log_int(16, 1024), rng.randint(1, 16), rng.choice([1, 40, 64, 80, 128])
        t = rng.choice(["bf16", "f32", "i32"])
        room = 1_600_000_000 // (heads * T * D * (2 if t == "bf16" else 4) * (K + n))      # what the largest listed case moves
        B = max(1, min(B, room))
        tensors = max(1, min(24, room // B))
        return dict(kind=kind, B=B, K=K, n=n, tensors=tensors, heads=heads, T=T, D=D, t=t,
                    ragged=rng.random() < 0.5)
    ended, first = rng.choice([0, 0, min(1, K - 1)]), rng.random() < 0.2
    if kind == "select":
        return dict(kind=kind, V=V, B=B, K=K, n=n, z=rng.choice(["f32", "bf16", "f16"]), ended=ended, first=first)
    B = max(1, min(B, 256 * 32000 * 5120 // (V * d * K)))
    return dict(kind=kind, V=V, d=d, B=B, K=K, n=n, ended=ended, first=first)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _head(V, d, g):
    """An LM head in 8 bits: rows of d integers at a pitch that is a multiple of 16, and a scale for each row."""
    W = _rand(g, V, d) * HEAD_STD
    top = W.abs().amax(1, keepdim=True)
    Wq = torch.zeros((V, (d + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    Wq[:, :d] = torch.round(W * (127.0 / top)).to(torch.int8)
    return Wq, (top[:, 0] / 127.0).contiguous()


def _beams(case, g):
    """Scores of the beams as a decoder has them, best first; some beams ended; at the first token one beam lives."""
    B, K = case["B"], case["K"]
    score = -3.0 - torch.cumsum(torch.rand((B, K), generator=g, device="cuda") * 2.0, 1)
    ended = torch.zeros((B, K), dtype=torch.uint8, device="cuda")
    if case["first"]:
        score[:, 1:] = -math.inf
        score[:, 0] = 0.0
    elif case["ended"]:
        at = torch.rand((B, K), generator=g, device="cuda").argsort(1)[:, :case["ended"]]
        ended.scatter_(1, at, 1)
    return score, ended


def _distinct(case):
    return max(1, min(case["n"], (3 * case["K"] + 4) // 5))


def _parents(case, g):
    """Of K beams about three in five have children; every one of them at least one, the rest of the n at random."""
    B, K, n, u = case["B"], case["K"], case["n"], _distinct(case)
    chosen = torch.rand((B, K), generator=g, device="cuda").argsort(1)[:, :u]
    more = torch.randint(0, u, (B, n - u), generator=g, device="cuda")
    pick = torch.cat([torch.arange(u, device="cuda").expand(B, u), more], 1)
    pick = pick.gather(1, torch.rand((B, n), generator=g, device="cuda").argsort(1))
    return chosen.gather(1, pick).to(torch.int32).contiguous()


def _lengths(case):
    """Positions in use, T down to about T / 2."""
    return [case["T"] - (b * case["T"]) // (2 * case["B"]) for b in range(case["B"])]


def prepare(case, seed):
    kind, g = case["kind"], _gen(seed)
    i32, f32, u8 = torch.int32, torch.float32, torch.uint8
    st = dict(case=case)

    def out(shape, dtype):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    V, d, rows = case.get("V", 8), case.get("d", 8), case["R"] if kind == "project" else case["B"] * case["K"]
    if kind in ("project", "step"):
        st["Wq"], st["w_scale"] = _head(V, d, g)
        st["H"] = _rand(g, rows, d).to(TYPES[case.get("x", "bf16")])
    if kind == "project":
        st["y"] = out((rows, V), TYPES[case["y"]])
    if kind == "reorder":
        B, K, n = case["B"], case["K"], case["n"]
        shape, t = (case["heads"], case["T"], case["D"]), case["t"]

        def states(rows):
            if t == "i32":
                return torch.randint(0, 32000, (rows, *shape), generator=g, device="cuda", dtype=i32)
            return _rand(g, rows, *shape).to(TYPES[t])

        st.update(parent=_parents(case, g), src=[states(B * K) for _ in range(case["tensors"])],
                  dst=[states(B * n) for _ in range(case["tensors"])], lens=None)
        if case["ragged"]:
            order = torch.rand(B, generator=g, device="cuda").argsort()
            st["lens"] = torch.tensor(_lengths(case), dtype=i32, device="cuda")[order].contiguous()
    if kind in ("select", "step"):
        B, K, n = case["B"], case["K"], case["n"]
        st["score"], st["ended"] = _beams(case, g)
        if kind == "select":   # logits of a head like the target's: independent, of a spread of 1.4
            st["logits"] = (_rand(g, B * K, V) * 1.4).to(TYPES[case["z"]])
        else:
            st["work"] = out((rows, V), f32)
        st.update(score_out=out((B, n), f32), parent=out((B, n), i32), token=out((B, n), i32), ended_out=out((B, n), u8))
    if own:
        from paper_2405_04304_b200 import binding
        st["ctx"] = binding.Context(V, d, d, max_batch=case.get("B", 1), max_rows=rows)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st, kind)
    if kind == "project":
        return _project(st["H"], st["Wq"], st["w_scale"], torch.float32).to(st["y"].dtype)
    if kind == "select":
        return _select(st["logits"], st["score"], st["ended"], st["case"]["n"])
    if kind == "step":
        z = _project(st["H"], st["Wq"], st["w_scale"], torch.float64)
        return _select(z, st["score"], st["ended"], st["case"]["n"])
    return _reorder(st["src"], st["dst"], st["parent"], st["lens"], st["case"]["K"])


def _own(st, kind):
    ctx = st["ctx"]
    if kind == "project":
        ctx.project_int8(st["Wq"], st["w_scale"], st["H"], st["y"])
        return st["y"]
    if kind == "reorder":
        ctx.beam_reorder(st["src"], st["dst"], st["parent"], lens=st["lens"], length_dim=2)
        return st["dst"]
    if kind == "select":
        ctx.beam_select(st["logits"], st["score"], st["score_out"], st["parent"], st["token"], finished=st["ended"], eos=EOS,
                        finished_out=st["ended_out"])
    else:
        ctx.beam_step_int8(st["Wq"], st["w_scale"], st["H"], st["score"], st["score_out"], st["parent"], st["token"],
                           st["work"], finished=st["ended"], eos=EOS, finished_out=st["ended_out"])
    return st["score_out"], st["parent"], st["token"], st["ended_out"]


# ------------------------------------------------------------------------------------------------ plain forms
def _project(H, Wq, w_scale, sums):
    """A scale for each hidden row from its largest number; integers by rounding to the nearest, ties to even (in 64 bits: a number
    on the border between two integers goes where it belongs); sums of products in `sums`, then both scales, in 32 bits."""
    x = H.double()
    top = x.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(x * 127.0 / top), torch.zeros_like(x))
    s = (top / 127.0).float()     # (a quotient by a number is a product with its reciprocal on the GPU: in 64 bits, too)
    acc = q.to(sums) @ Wq[:, :H.shape[1]].to(sums).T
    return acc.float() * s * w_scale


def _select(z, score, ended, n):
    """Scores in 64 bits: which of two near ones is the better decides a whole number."""
    B, K = score.shape
    z = z.double().view(B, K, -1)
    V = z.shape[2]
    top = z.amax(2, keepdim=True)
    l = score.double()[:, :, None] + (z - (top + (z - top).exp().sum(2, keepdim=True).log()))
    eos = torch.arange(V, device=z.device) == EOS
    l = torch.where(ended[:, :, None] != 0, torch.where(eos, score.double()[:, :, None], -math.inf), l)
    l = torch.where(score[:, :, None] > -math.inf, l, -math.inf)
    best, at = torch.sort(l.view(B, K * V), dim=1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    none = best == -math.inf
    parent, token = torch.where(none, -1, at // V), torch.where(none, -1, at % V)
    over = (ended.gather(1, parent.clamp_min(0)) != 0) | (token == EOS)
    return best.float(), parent.to(torch.int32), token.to(torch.int32), (over & ~none).to(torch.uint8)


def _reorder(src, dst, parent, lens, K):
    B, n = parent.shape
    at = (torch.arange(B, device=parent.device)[:, None] * K + parent).view(-1)
    if lens is None:
        return [s[at] for s in src]
    keep = torch.arange(src[0].shape[2], device=parent.device) < lens.repeat_interleave(n)[:, None]
    return [torch.where(keep[:, None, :, None], s[at], t) for s, t in zip(src, dst)]


# ------------------------------------------------------------------------------------------------ by definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "reorder":
        K, n, got = case["K"], case["n"], [t.to(torch.float64) if t.is_floating_point() else t.clone() for t in st["dst"]]
        used = st["lens"].tolist() if case["ragged"] else [case["T"]] * case["B"]
        for b, children in enumerate(st["parent"].tolist()):
            for j, k in enumerate(children):
                for s, t in zip(st["src"], got):
                    t[b * n + j, :, :used[b]] = s[b * K + k, :, :used[b]]
        return got
    if kind in ("project", "step"):
        x = st["H"].to(torch.float64)
        f = x.abs().max(dim=1, keepdim=True).values
        q = torch.div(127 * x, torch.where(f > 0, f, 1.0)).round()
        z = torch.einsum("rk,vk->rv", q, st["Wq"][:, :case["d"]].to(torch.float64))
        z = z * st["w_scale"].to(torch.float64)[None, :] * (f / 127.0)
        if kind == "project":
            return z
    else:
        z = st["logits"].to(torch.float64)
    B, K, V, n = case["B"], case["K"], case["V"], case["n"]
    logp = z.reshape(B, K, V) - torch.logsumexp(z, 1).reshape(B, K, 1)
    logp += st["score"].to(torch.float64).reshape(B, K, 1)
    for b, k in (st["ended"] != 0).nonzero().tolist():
        logp[b, k] = -math.inf
        logp[b, k, EOS] = float(st["score"][b, k])
    logp[(st["score"] == -math.inf)] = -math.inf
    score = torch.full((B, n), -math.inf, dtype=torch.float64, device="cuda")
    parent, token = torch.full((B, n), -1, dtype=torch.int32, device="cuda"), torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    over = torch.zeros((B, n), dtype=torch.uint8, device="cuda")
    for b in range(B):   # all that are as good as the n-th best, lowest places first; then by value
        row = logp[b].reshape(-1)
        at = ((row >= torch.topk(row, min(n, K * V)).values[-1]) & (row > -math.inf)).nonzero().flatten()
        at = at[torch.argsort(-row[at], stable=True)][:n]
        m = at.numel()
        score[b, :m], parent[b, :m], token[b, :m] = row[at], (at // V).to(torch.int32), (at % V).to(torch.int32)
        over[b, :m] = ((st["ended"][b][at // V] != 0) | (at % V == EOS)).to(torch.uint8)
    return score, parent, token, over


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    """The 8-bit head and its scales, the hidden rows and the logits of live beams read once, what is returned written once; states:
    every row that has a child read once, every child written.  Two operations per multiply-add."""
    kind = case["kind"]
    size = {"f32": 4, "i32": 4, "bf16": 2, "f16": 2}
    if kind == "project":
        V, d, R = case["V"], case["d"], case["R"]
        return dict(bytes=V * (d + 4) + size[case["x"]] * R * d + size[case["y"]] * R * V, flops=2 * R * V * d)
    B, K, n = case["B"], case["K"], case["n"]
    if kind == "reorder":
        positions = sum(_lengths(case)) if case["ragged"] else B * case["T"]
        row = case["heads"] * case["D"] * size[case["t"]]
        return dict(bytes=case["tensors"] * positions * row * (_distinct(case) + n) + 4 * B * n, flops=0)
    live = B if case["first"] else B * (K - case["ended"])
    ends = 5 * B * K + 13 * B * n
    if kind == "select":
        return dict(bytes=size[case["z"]] * live * case["V"] + ends, flops=4 * live * case["V"])
    V, d = case["V"], case["d"]
    return dict(bytes=V * (d + 4) + 2 * live * d + ends, flops=2 * live * V * d)
