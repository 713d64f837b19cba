"""Beam selection against the definition of include/lora_abi.h in 64 bits, and what the calls refuse.

Tolerance, derived: an exponential is off by at most 2^-22 of itself (exp2 of the hardware 2^-23, its argument's rounding carried on to 2^-30,
the last product 2^-24), all others are sums in 64 bits, so a row's log sum is off by at most 2^-22; a score is rounded once, 2^-24 of it.
Candidates whose worth in 64 bits differs by more than twice 2^-22 have to come in that order."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B

DEV = "cuda:0"
gpu = pytest.mark.gpu
BF16, F32 = B.LORA_BF16, B.LORA_F32
TORCH = {BF16: torch.bfloat16, F32: torch.float32}
NEAR = 2.0 ** -21


def worth(x, score, ended, end):
    """Of every (beam, token) of a request, -inf where there is no continuation.  x [beams, vocab] in float32 values"""
    x = x.astype(np.float64)
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        lse = np.log(np.exp(x - top).sum(-1, keepdims=True)) + top
        c = score.astype(np.float64)[:, None] + (x - lse)
    c[~np.isfinite(lse[:, 0]) | ~np.isfinite(score)] = -np.inf
    for b in np.flatnonzero(ended):
        c[b] = -np.inf
        if np.isfinite(score[b]):
            c[b, end] = score[b]
    return c


def run(x, score, last, end, beams, out, dtype, pad=0, shift=0, stream=None):
    rows, vocab = x.shape
    groups, ld = rows // beams, vocab + pad
    buf = torch.full((rows * ld + shift,), float("nan"), dtype=TORCH[dtype], device=DEV)
    view = buf[shift:].view(rows, ld)
    view[:, :vocab] = torch.from_numpy(x).to(TORCH[dtype]).to(DEV)
    sd = torch.from_numpy(score.astype(np.float32)).to(DEV)
    ldv = None if last is None else torch.from_numpy(last.astype(np.int32)).to(DEV)
    got = [torch.full((groups * out + 2,), -9, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    need = B.lora_beam_workspace(groups, beams, vocab, out)
    room = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    B.lora_beam_select(dtype, groups, beams, vocab, view, ld, sd, ldv, end, out, *got, room, need, stream=stream)
    torch.cuda.synchronize()
    assert all((g[-2:] == -9).all() for g in got)
    return [g[:-2].cpu().numpy().reshape(groups, out) for g in got]


def check(x, score, last, end, beams, out, dtype, exact=False, **layout):
    x = torch.from_numpy(np.asarray(x, np.float32)).to(TORCH[dtype]).float().numpy()
    s, parent, token = run(x, score, last, end, beams, out, dtype, **layout)
    vocab = x.shape[1]
    for g in range(len(x) // beams):
        r = slice(g * beams, (g + 1) * beams)
        ended = np.zeros(beams, bool) if last is None or end < 0 else last[r] == end
        with np.errstate(all="ignore"):
            c = worth(x[r], score[r], ended, end)
        flat = c.ravel()
        # equal ones by beam, logit, token
        key = np.where(np.isnan(x[r]), -np.inf, x[r]).ravel()
        order = np.lexsort((np.arange(flat.size), -key, np.repeat(np.arange(beams), vocab), -flat))[:out]
        order = order[flat[order] > -np.inf]
        n = len(order)
        assert (parent[g, n:] == -1).all() and (token[g, n:] == -1).all() and (s[g, n:] == -np.inf).all(), g
        at = (parent[g, :n] - g * beams) * vocab + token[g, :n]
        assert ((parent[g, :n] >= g * beams) & (parent[g, :n] < (g + 1) * beams) & (token[g, :n] >= 0) & (token[g, :n] < vocab)).all()
        assert len(set(at.tolist())) == n
        assert np.all(np.abs(flat[at] - flat[order]) <= NEAR), (g, flat[at], flat[order])
        assert np.all(np.abs(s[g, :n] - flat[at]) <= 2.0 ** -22 + 2.0 ** -24 * np.abs(flat[at])), g
        # where nothing of another beam is near, it is that one
        for i in range(n):
            near = np.flatnonzero(np.abs(flat - flat[order[i]]) <= NEAR)
            if exact or len(set((near // vocab).tolist())) == 1:
                assert at[i] == order[i], (g, i, divmod(at[i], vocab), divmod(order[i], vocab))
    return s, parent, token


def logits(rng, rows, vocab, spread=2.0):
    x = rng.standard_normal((rows, vocab)).astype(np.float32) * np.float32(spread)
    for r in range(rows):
        some = rng.integers(0, vocab, 20)
        x[r, some] += 7 + 2 * rng.standard_normal(20).astype(np.float32)
    return x


def scores(rng, rows):
    return (-4 - 6 * rng.random(rows)).astype(np.float32)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,beams,vocab,out", [(1, 1, 1, 1), (1, 1, 1, 7), (2, 3, 2, 64), (1, 4, 32000, 8), (3, 5, 2049, 10), (5, 2, 8191, 4), (2, 16, 4097, 32), (1, 64, 700, 64), (40, 2, 300, 2),
                                                    (70, 8, 9000, 16), (1, 1, 100001, 64), (130, 4, 16500, 1)])
def test_selection(dtype, groups, beams, vocab, out):
    rng = np.random.default_rng(vocab + out)
    rows = groups * beams
    last = rng.integers(0, vocab, rows)
    last[rng.random(rows) < 0.2] = vocab // 2
    check(logits(rng, rows, vocab), scores(rng, rows), last, vocab // 2, beams, out, dtype)
    check(logits(rng, rows, vocab), scores(rng, rows), None, 0, beams, out, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (3, 3), (8, 8), (5, 2)])
@pytest.mark.parametrize("vocab", [1000, 20011])
def test_rows_of_any_layout(dtype, pad, shift, vocab):
    rng = np.random.default_rng(pad + shift)
    check(logits(rng, 12, vocab), scores(rng, 12), None, 0, 4, 8, dtype, pad=pad, shift=shift)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [64, 5000, 70000])
@pytest.mark.parametrize("groups", [1, 150])
def test_equal_logits_go_by_beam_and_token(dtype, vocab, groups):
    """All equal; a few values; equal rows of equal scores: whole numbers, whose sums are the same for equal rows"""
    rng, beams, out = np.random.default_rng(vocab), 4, 16
    rows = groups * beams if vocab < 70000 else beams
    check(np.zeros((rows, vocab)), np.zeros(rows, np.float32), None, 0, beams, out, dtype, exact=True)
    row = rng.integers(0, 3, vocab).astype(np.float32)
    check(np.tile(row, (rows, 1)), np.full(rows, -2, np.float32), None, 0, beams, out, dtype, exact=True)
    check(rng.integers(0, 2, (rows, vocab)), scores(rng, rows), None, 0, beams, out, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_first_step_has_one_beam(dtype):
    """Beams that are not there yet have the score -inf; others' scores that are no number give nothing either"""
    rng, beams = np.random.default_rng(2), 4
    x = logits(rng, 3 * beams, 3000)
    score = np.array([0, -np.inf, -np.inf, -np.inf, np.nan, np.inf, -1, -np.inf, -np.inf, -np.inf, -np.inf, -np.inf], np.float32)
    _, parent, _ = check(x, score, None, 0, beams, 8, dtype)
    assert (parent[0] == 0).all() and (parent[1] == 6).all() and (parent[2] == -1).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [50, 9000])
def test_masked_tokens_and_rows(dtype, vocab):
    """-inf in most places, in whole pieces of a row, in whole rows; the type's lowest value; NaN and +inf in a row"""
    rng, beams, out = np.random.default_rng(7), 5, 12
    x = logits(rng, 6 * beams, vocab)
    low = float(torch.finfo(TORCH[dtype]).min)
    x[0:5, : vocab * 9 // 10] = -np.inf
    x[5:9] = -np.inf                                        # one beam is left, with three tokens
    x[9, 3:] = -np.inf
    x[10:15, ::2] = low
    x[15:20] = low                                          # (all equal)
    x[16, vocab // 3] = np.nan
    x[17, vocab - 1] = np.inf
    x[20:25] = -np.inf
    x[25:30, 1:] = -np.inf
    s, parent, token = check(x, scores(rng, len(x)), None, 0, beams, out, dtype)
    assert (token[1, :3] >= 0).all() and (token[1, 3:] == -1).all() and (parent[4] == -1).all()
    assert not np.isin(parent[3], (16, 17)).any() and (token[3, :out] >= 0).all()
    assert sorted(parent[5][:5].tolist()) == [25, 26, 27, 28, 29] and (token[5, :5] == 0).all() and (token[5, 5:] == -1).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_up_to_the_end_of_their_range(dtype):
    rng, beams = np.random.default_rng(8), 3
    top = float(torch.finfo(TORCH[dtype]).max)
    x = rng.standard_normal((9, 5000)).astype(np.float32)
    x[0:3] *= 1e30
    x[3, 4000:4003], x[4, 7], x[5] = top, top, -top
    x[6:9] = x[6:9] * 1e-40 - 3
    x[7, 100:] = -1e30
    check(x, scores(rng, 9), None, 0, beams, 6, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ended_beams_stay(dtype):
    rng, beams, vocab, end = np.random.default_rng(9), 4, 6000, 5999
    x, score = logits(rng, 12, vocab), scores(rng, 12)
    x[1] = np.nan                                           # (a row that has ended is not looked at)
    last = rng.integers(0, 5000, 12)
    last[[1, 4, 5, 6, 7, 8]] = end
    score[8] = -np.inf
    s, parent, token = check(x, score, last, end, beams, 8, dtype)
    order = np.argsort(-score[4:8], kind="stable")
    assert (token[1, :4] == end).all() and parent[1, :4].tolist() == (4 + order).tolist() and s[1, :4].tolist() == score[4:8][order].tolist()
    assert (token[1, 4:] == -1).all() and not (parent[2] == 8).any()
    x[1] = 0
    check(x, score, last, -1, beams, 8, dtype)              # nothing ends
    last[:] = -1
    check(x, score, last, -1, beams, 8, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,vocab", [(2, 9000), (40, 65536 + 77)])
@pytest.mark.parametrize("order", ["up", "down", "close", "close up", "steps", "late", "few"])
@pytest.mark.parametrize("out", [5, 64])
def test_orders_of_logits_that_bounds_do_not_help(dtype, groups, vocab, order, out):
    """Growing and falling along the row; within one step of 16 bits of each other; equal in long runs; the first half masked; all but a few masked"""
    rng, beams = np.random.default_rng(out), 4
    rows, i = groups * beams, np.arange(vocab)
    if order in ("up", "down"):
        x = np.tile(i * 1e-3 * (1 if order == "up" else -1), (rows, 1)) + 0.3 * rng.random((rows, 1))
    elif order.startswith("close"):
        x = 1 + (i % 8191 if order == "close up" else rng.integers(0, 8191, (rows, vocab))) * 2.0 ** -21 + 0 * rng.random((rows, 1))
    elif order == "steps":
        x = np.floor(i / 3000) % 5 + 0 * rng.random((rows, 1))
    else:
        x = logits(rng, rows, vocab)
        x[:, :vocab // 2] = -np.inf
        if order == "few":
            x[:, rng.permutation(vocab)[:vocab - 70]] = -np.inf
    check(np.asarray(x, np.float32), scores(rng, rows), None, 0, beams, out, dtype)


@gpu
def test_the_largest_vocabulary():
    vocab = 1 << 24
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.randn((2, vocab), generator=gen, device=DEV)
    x[0, vocab - 1], x[1, 0], x[1, 9000000] = 30.0, 29.0, 29.0
    score = torch.tensor([-1.0, -0.5], device=DEV)
    out = [torch.empty(5, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    need = B.lora_beam_workspace(1, 2, vocab, 5)
    B.lora_beam_select(F32, 1, 2, vocab, x, vocab, score, None, 0, 5, *out, torch.empty(need, dtype=torch.uint8, device=DEV), need)
    c = torch.log_softmax(x.double(), -1) + score.double()[:, None]
    best = torch.sort(c.flatten(), descending=True, stable=True)
    assert (out[1].long() * vocab + out[2]).tolist() == best.indices[:5].tolist()
    assert (out[0].double() - best.values[:5]).abs().max() <= 2.0 ** -22 + 2.0 ** -24 * 20


@gpu
def test_rows_beyond_4_gb():
    vocab, ld, beams = 3000, (3 << 30) // 2 // 3, 4                # (row 3 begins 3 GB on, and it ends there)
    rng = np.random.default_rng(10)
    x = torch.from_numpy(logits(rng, beams, vocab)).bfloat16()
    buf = torch.zeros((beams - 1) * ld + vocab, dtype=torch.bfloat16, device=DEV)
    for b in range(beams):
        buf[b * ld:b * ld + vocab] = x[b].to(DEV)
    score = torch.zeros(beams, device=DEV)
    out = [torch.empty(6, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    need = B.lora_beam_workspace(1, beams, vocab, 6)
    B.lora_beam_select(BF16, 1, beams, vocab, buf, ld, score, None, 0, 6, *out, torch.empty(need, dtype=torch.uint8, device=DEV), need)
    a = [o.cpu().numpy() for o in out]
    b = run(x.float().numpy(), np.zeros(beams), None, 0, beams, 6, BF16)
    assert all(np.array_equal(p, q[0]) for p, q in zip(a, b))


@gpu
def test_a_captured_selection_on_a_stream_of_its_own():
    rng, groups, beams, vocab, out = np.random.default_rng(3), 3, 4, 12000, 4
    rows = groups * beams
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device=DEV)
    score, last = torch.zeros(rows, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    got = [torch.empty((groups, out), dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    need = B.lora_beam_workspace(groups, beams, vocab, out)
    room = torch.empty(need, dtype=torch.uint8, device=DEV)
    call = lambda: B.lora_beam_select(BF16, groups, beams, vocab, x, vocab, score, last, 5, out, *got, room, need)  # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        values, s, l = logits(rng, rows, vocab), scores(rng, rows), rng.integers(0, 9, rows)
        x.copy_(torch.from_numpy(values))
        score.copy_(torch.from_numpy(s))
        last.copy_(torch.from_numpy(l.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [g.cpu().numpy() for g in got]
        eager = check(values, s, l, 5, beams, out, BF16)
        assert all(np.array_equal(a, b) for a, b in zip(replayed, eager))
        torch.ones(1000, device=DEV).sum()


# ---- refusals (no GPU) ---------------------------------------------------------------------------------------------------
def status(call):
    try:
        call()
    except B.LoraError as e:
        return e.status
    return B.LORA_OK


def test_calls_are_refused():
    need = B.lora_beam_workspace(4, 5, 1000, 10)
    MB = 1 << 20
    fine = dict(dtype=BF16, num_groups=4, beams=5, vocab=1000, logits=MB, ld=1000, d_score=2 * MB, d_last_token=3 * MB, end_token=2, num_out=10, d_out_score=4 * MB,
                d_out_parent=5 * MB, d_out_token=6 * MB, workspace=7 * MB, workspace_bytes=need)
    call = lambda **f: status(lambda: B.lora_beam_select(**{**fine, **f}, stream=1))  # noqa: E731
    for f in (dict(dtype=2), dict(num_groups=-1), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25), dict(num_out=0), dict(num_out=65),
              dict(end_token=1 << 24), dict(ld=999), dict(logits=None), dict(logits=MB + 1), dict(d_score=None), dict(d_score=2 * MB + 2), dict(d_last_token=3 * MB + 1),
              dict(d_out_score=None), dict(d_out_parent=None), dict(d_out_token=None), dict(d_out_score=4 * MB + 2), dict(d_out_parent=5 * MB + 2), dict(d_out_token=6 * MB + 1),
              dict(dtype=F32, logits=MB + 2)):
        assert call(**f) == B.LORA_ERR_INVALID_ARG, f
    # outputs on inputs, on each other, on the workspace
    for f in (dict(d_out_score=2 * MB), dict(d_out_token=3 * MB + 76), dict(d_out_parent=4 * MB + 156), dict(d_out_score=MB + 20 * 2000 - 4), dict(d_out_token=7 * MB + need - 4),
              dict(workspace=MB - 256), dict(workspace=2 * MB), dict(d_out_parent=MB - 156)):
        assert call(**f) == B.LORA_ERR_INVALID_ARG, f
    for f in (dict(workspace=None), dict(workspace=7 * MB + 64), dict(workspace_bytes=need - 1)):
        assert call(**f) == B.LORA_ERR_WORKSPACE, f
    for f in (dict(num_groups=1 << 29, beams=4), dict(num_groups=1 << 23, beams=2), dict(ld=1 << 59)):
        assert call(**f) == B.LORA_ERR_UNSUPPORTED, f
    assert call(num_groups=0, logits=None) == B.LORA_OK and B.lora_beam_workspace(0, 4, 100, 4) == 0
    with pytest.raises(B.LoraError):
        B.lora_beam_workspace(1, 0, 100, 4)


def test_the_workspace_holds_every_piece():
    """Sums of 16 bytes and num_out candidates of 8 for every piece of a row: 2048 tokens, or as many times 4096 as leave four pieces a compute unit"""
    for groups, beams, vocab, out, pieces in ((1, 1, 1, 1, 1), (1, 4, 32000, 8, 16), (64, 8, 131072, 16, 2), (100, 6, 8192, 3, 2), (100, 6, 8193, 64, 3), (1000, 2, 20000, 4, 1),
                                              (64, 4, 50021, 4, 5), (600, 1, 4095, 7, 2)):
        pieces *= groups * beams
        assert B.lora_beam_workspace(groups, beams, vocab, out) == -(-(-(-pieces * 16 // 256) * 256 + pieces * out * 8) // 256) * 256, (groups, beams, vocab)


def test_the_definition_by_hand():
    x = np.array([[0, 0, 0, 0], [np.log(2), 0, 0, -np.inf]], np.float32)
    c = worth(x, np.float32([-1, -2]), np.array([False, False]), 0)
    assert np.allclose(c[0], -1 - np.log(4)) and np.allclose(c[1, :3], [-2 - np.log(2), -2 - np.log(4), -2 - np.log(4)]) and c[1, 3] == -np.inf
    c = worth(x, np.float32([-1, -np.inf]), np.array([True, True]), 3)
    assert c[0].tolist() == [-np.inf] * 3 + [-1] and (c[1] == -np.inf).all()
