"""Bounds of a page's keys, the choice of pages by them and attention over the chosen ones, against the definitions of include/lora_abi.h, and what the
calls refuse.  Bounds and choices are whole numbers (the definitions round what is no whole number in 32 bits, as numpy does) and have
to be equal; the attention's tolerance is that of test_attention.py, over the slots that are seen."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B
from test_attention import BF16, DEV, F32, TORCH, Pool, check, gpu, held, offsets, padded, quantised, reference, rounded, to_device, tokens

F = np.float32
THIRD = F(1) / F(127)


# ---- definitions ---------------------------------------------------------------------------------------------------------
def bounds_of(k):
    """Of the keys [tokens, D] (float32 values that a page holds): upper, lower, step"""
    with np.errstate(all="ignore"):
        most = np.abs(k).max()
        if not most < np.inf:                               # (NaN among them)
            return np.zeros(k.shape[1], np.int8), np.zeros(k.shape[1], np.int8), F("nan")
        step = F(most * THIRD)
        if step < 2.0 ** -100:
            return np.zeros(k.shape[1], np.int8), np.zeros(k.shape[1], np.int8), F(0)
        up, down = np.ceil(k.max(0) / step), np.floor(k.min(0) / step)
        return np.minimum(up, 127).astype(np.int8), np.maximum(down, -127).astype(np.int8), step


def codes_of(q):
    """Codes and unit of a query [D]"""
    with np.errstate(all="ignore"):
        if not np.isfinite(q).all():
            return np.zeros(len(q), np.int64), F("nan")
        unit = F(np.abs(q).max() * THIRD)
        if unit < 2.0 ** -100:
            return np.zeros(len(q), np.int64), F(0)
        return np.clip(np.rint(q / unit), -127, 127).astype(np.int64), unit


def choice(q, upper, lower, steps, there, budget, first, recent):
    """q [group, D]; upper, lower [pages, D], steps [pages] of the pages that the token sees; there: which of them are"""
    m = len(steps)
    if m <= budget:
        return [p for p in range(m) if there[p]]
    best = None
    for h in range(len(q)):
        c, unit = codes_of(q[h])
        s = (upper.astype(np.int64) @ np.maximum(c, 0) + lower.astype(np.int64) @ np.minimum(c, 0)).astype(F) * unit
        best = s if best is None else np.maximum(best, s)   # (NaN goes on)
    score = best * steps
    always = [p for p in range(m) if there[p] and (p < first or p >= m - recent)]
    rest = [p for p in range(m) if there[p] and p not in set(always)]
    rest.sort(key=lambda p: (not np.isnan(score[p]), -score[p] if not np.isnan(score[p]) else 0, p))
    return sorted(always + rest[:budget - len(always)])


def digest(pool, new=None, max_new=None, lengths=None, bounds=None, steps=None):
    """Call and result; new: tokens of every sequence (None: one each, without offsets)"""
    bounds = torch.full((pool.n, pool.Hkv, 2, padded(pool.D)), 99, dtype=torch.int8, device=DEV) if bounds is None else bounds
    steps = torch.full((pool.n, pool.Hkv), -5.0, device=DEV) if steps is None else steps
    ptr = None if new is None else torch.from_numpy(offsets(new)).to(DEV)
    n = len(pool.table) if new is None else sum(new)
    B.lora_cache_digest(pool.cache, n, (1 if new is None else max(new)) if max_new is None else max_new, ptr, bounds, steps)
    torch.cuda.synchronize()
    return bounds, steps


def held_keys(vals):
    """What the cache holds, in the 32 bits that lora_cache_read gives: keys [length, Hkv, D]"""
    c, step, zero = quantised(vals[0])
    with np.errstate(all="ignore"):
        return (c.astype(F) * step[..., None]).astype(F) + zero[..., None]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,page,Hkv", [(64, 32, 3), (128, 64, 2), (80, 96, 1), (256, 32, 2), (33, 64, 5), (1, 32, 1), (100, 1024, 1)])
@pytest.mark.parametrize("new", [0, 1, 70])
def test_bounds(dtype, D, page, Hkv, new):
    """Of all tokens, single ones, several: pages that end inside, sequences without tokens, pages that are not there; nothing else is written"""
    rng = np.random.default_rng(D + new)
    lengths = [1, 0, 33, page, 2 * page + 5, 130, 64]
    pool = Pool(lengths, Hkv, D, page, seed=D, missing=((5, 0), (4, 1)))
    vals = tokens(rng, lengths, Hkv, D, dtype)
    for s in (2, 6):
        vals[s][0][: min(3, lengths[s])] = 0                # (a step of 0 among tokens)
    vals[6][0][:] = 0
    if page > 32:
        vals[5][0][lengths[5] - 1, 0, 0] = np.nan
    pool.fill(vals, dtype)
    count = [n if new == 0 else min(n, new) for n in lengths]
    bounds, steps = (x.cpu().numpy() for x in digest(pool, None if new == 1 and 0 not in lengths else count))
    expect, unit = np.full(bounds.shape, 99, np.int8), np.full(steps.shape, -5, F)
    for s, (n, m) in enumerate(zip(lengths, count)):
        k = held_keys(vals[s])
        for p in range((n - m) // page if m else n, -(-n // page)):
            if not pool.there(s, p * page):
                continue
            at = pool.table[s, p]
            for h in range(Hkv):
                up, down, unit[at, h] = bounds_of(k[p * page:(p + 1) * page, h])
                expect[at, h] = 0
                expect[at, h, 0, :D], expect[at, h, 1, :D] = up, down
    assert np.array_equal(steps, unit, equal_nan=True)
    assert np.array_equal(bounds, expect)
    # bounds they are
    for s, n in enumerate(lengths):
        k = held_keys(vals[s])
        for p in range(-(-n // page)):
            at = pool.table[s, p]
            if pool.there(s, p * page) and steps[at, 0] > 0:
                x, u = k[p * page:(p + 1) * page, 0].astype(np.float64), float(steps[at, 0])
                slack = u * 127 * 2.0 ** -22                # (the step and the quotient were rounded: 2^-24 each of at most 127)
                assert (x <= bounds[at, 0, 0, :D] * u + slack).all() and (x >= bounds[at, 0, 1, :D] * u - slack).all()


@gpu
def test_bounds_of_single_tokens_without_offsets_and_of_no_more_than_the_call_says():
    rng, D = np.random.default_rng(1), 64
    lengths = [33, 64, 200]
    pool = Pool(lengths, 2, D, 32)
    vals = tokens(rng, lengths, 2, D, BF16)
    pool.fill(vals)
    a = digest(pool)
    b = digest(pool, [1, 1, 1])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # of 100 tokens of the last sequence the first 10 are taken: slots 100 .. 109
    bounds, steps = digest(pool, [0, 0, 100], max_new=10)
    touched = {int(pool.table[2, 3])}
    assert {int(p) for p in (steps[:, 0] != -5).nonzero()} == touched


@gpu
def test_values_at_the_end_of_their_range_and_below_the_normal_numbers():
    rng, D = np.random.default_rng(1), 64
    lengths = [30, 30, 30, 30]
    pool = Pool(lengths, 1, D, 32)
    vals = [[(rng.standard_normal((30, 1, D)) * x).astype(F) for _ in range(2)] for x in (1e37, 1e-30, 1e-38, 1e-44)]
    pool.fill(vals)
    bounds, steps = (x.cpu().numpy() for x in digest(pool, lengths))
    for s in range(4):
        up, down, unit = bounds_of(held_keys(vals[s])[:, 0])
        at = pool.table[s, 0]
        assert np.array_equal(bounds[at, 0, 0], up) and np.array_equal(bounds[at, 0, 1], down) and steps[at, 0] == unit


# ---- the choice ----------------------------------------------------------------------------------------------------------
def run_choose(pool, q, new, dtype, bounds, steps, budget, first, recent, ptr="given", pad=0, shift=0):
    H, D = q.shape[1], q.shape[2]
    width = H * D + pad
    buf = torch.full((len(q) * width + shift,), float("nan"), dtype=TORCH[dtype], device=DEV)
    qd = buf[shift:].view(len(q), width)
    qd[:, :H * D] = to_device(q, dtype).view(len(q), H * D)
    out = torch.full((len(q) + 1, pool.Hkv, budget), -9, dtype=torch.int32, device=DEV)
    need = B.lora_cache_choose_workspace(pool.cache, len(q), max(new))
    room = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device=DEV)
    d_ptr = torch.from_numpy(offsets(new)).to(DEV) if ptr == "given" else None
    B.lora_cache_choose(pool.cache, dtype, H, len(q), max(new), d_ptr, qd, width, bounds, steps, budget, first, recent, out, room if need else None, need)
    torch.cuda.synchronize()
    assert (out[-1] == -9).all()
    return out[:-1]


def check_choice(pool, q, new, lengths, bounds, steps, budget, first, recent, got):
    b, u, got = bounds.cpu().numpy(), steps.cpu().numpy(), got.cpu().numpy()
    at, G = offsets(new), q.shape[1] // pool.Hkv
    for s, n in enumerate(new):
        for i in range(n):
            m = -(-max(0, lengths[s] - n + i + 1) // pool.page)
            there = [pool.there(s, p * pool.page) for p in range(m)]
            rows = np.where(there, pool.table[s, :m], 0).astype(int)
            for h in range(pool.Hkv):
                want = choice(q[at[s] + i, h * G:(h + 1) * G], b[rows, h, 0, :pool.D], b[rows, h, 1, :pool.D], u[rows, h], there, budget, first, recent)
                assert got[at[s] + i, h].tolist() == want + [-1] * (budget - len(want)), (s, i, h)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 128), (8, 2, 64), (5, 1, 80), (4, 2, 256), (24, 1, 33), (40, 1, 64)])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 0, 1), (5, 1, 2), (16, 0, 0), (7, 3, 4), (200, 1, 1)])
def test_pages_are_chosen(dtype, H, Hkv, D, budget, first, recent):
    """Sequences with fewer pages than the budget, with none, with one that is not there; several tokens, each with its own pages"""
    rng = np.random.default_rng(D + budget)
    lengths, new = [1, 0, 33, 700, 300, 2], [1, 0, 4, 3, 1, 4]
    pool = Pool(lengths, Hkv, D, 32, seed=H, missing=((4, 3), (4, 0), (3, 21)))
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    bounds, steps = digest(pool, lengths)
    q = rounded(rng.standard_normal((sum(new), H, D)), dtype)
    for layout in (dict(), dict(pad=3, shift=1)):
        got = run_choose(pool, q, new, dtype, bounds, steps, budget, first, recent, **layout)
        check_choice(pool, q, new, lengths, bounds, steps, budget, first, recent, got)


@gpu
@pytest.mark.parametrize("budget", [1, 10, 33])
def test_equal_pages_go_by_number_and_nan_is_above_all(budget):
    rng, D = np.random.default_rng(2), 64
    lengths = [32 * 40, 32 * 40, 32 * 40]
    pool = Pool(lengths, 1, D, 32)
    block = rng.standard_normal((32, 1, D)).astype(F)
    vals = [[np.tile(block, (40, 1, 1)), np.tile(block, (40, 1, 1))] for _ in lengths]
    vals[1][0][32 * 7: 32 * 8] *= 2
    vals[1][0][32 * 20, 0, 3] = np.inf
    vals[1][0][32 * 30, 0, 3] = np.nan
    vals[2][0][:] = 0
    pool.fill(vals)
    bounds, steps = digest(pool, lengths)
    q = rng.standard_normal((3, 2, D)).astype(F)
    for x in (q, np.zeros_like(q), np.where(np.arange(D) == 5, F("nan"), q), np.where(np.arange(D) == 5, F("inf"), q)):
        got = run_choose(pool, x.astype(F), [1, 1, 1], F32, bounds, steps, budget, 0, 1, ptr=None)
        check_choice(pool, x.astype(F), [1, 1, 1], lengths, bounds, steps, budget, 0, 1, got)
    assert budget == 1 or {20, 30} <= set(run_choose(pool, q, [1, 1, 1], F32, bounds, steps, 10, 0, 0, ptr=None)[1, 0].tolist())


class Long:
    """A cache whose sequences name the same few pages again and again: long tables over little memory"""

    def __init__(self, lengths, Hkv, D, page, pages, seed, max_length=None):
        rng = np.random.default_rng(seed)
        self.page, self.Hkv, self.D, self.n = page, Hkv, D, pages
        self.table = rng.integers(0, pages, (len(lengths), -(-max(*lengths, max_length or 1) // page))).astype(np.int32)
        self.pages = torch.zeros((pages, Hkv, B.lora_cache_page_bytes(page, D)), dtype=torch.uint8, device=DEV)
        self.length, self.d_table = torch.tensor(lengths, dtype=torch.int32, device=DEV), torch.from_numpy(self.table).to(DEV)
        self.cache = B.lora_cache(self.pages, self.d_table, self.length, page, Hkv, D, max_length or max(lengths))
        self.bounds = torch.from_numpy(rng.integers(-127, 128, (pages, Hkv, 2, padded(D))).astype(np.int8)).to(DEV)
        self.bounds[..., D:] = 0
        self.steps = torch.from_numpy(rng.random((pages, Hkv)).astype(F) + F(0.1)).to(DEV)

    def there(self, s, slot):
        return True


@gpu
@pytest.mark.parametrize("lengths,max_length,budget", [([32 * 12200, 5000], None, 100), ([32 * 12288], None, 3), ([32 * 12289 + 1, 40, 32 * 3000], None, 700), ([32 * 20000], None, 12000),
                                                       ([3000, 32], 32 * 50000, 30)])
def test_long_tables(lengths, max_length, budget):
    """Keys of the pages in LDS and, past what it holds, in the workspace; many equal ones, as a page is named often"""
    rng, D = np.random.default_rng(4), 64
    pool = Long(lengths, 2, D, 32, 300 if budget > 100 else 5000, 3, max_length)
    q = rng.standard_normal((len(lengths), 4, D)).astype(F)
    need = B.lora_cache_choose_workspace(pool.cache, len(lengths), 1)
    assert need > 0                                         # (few tokens: their pages' scores are of a launch of their own)
    got = run_choose(pool, q, [1] * len(lengths), F32, pool.bounds, pool.steps, budget, 1, 1, ptr=None)
    check_choice(pool, q, [1] * len(lengths), lengths, pool.bounds, pool.steps, budget, 1, 1, got)


# ---- attention -----------------------------------------------------------------------------------------------------------
def run_chosen(pool, q, new, dtype, scale, chosen, ptr="given", pad=0, shift=0):
    H, D = q.shape[1], q.shape[2]
    width, budget = H * D + pad, chosen.shape[2]
    buf = torch.zeros(len(q) * width + shift, dtype=TORCH[dtype], device=DEV)
    qd = buf[shift:].view(len(q), width)
    qd[:, :H * D] = to_device(q, dtype).view(len(q), H * D)
    out = torch.full((len(q) + 1, width), -7.0, dtype=TORCH[dtype], device=DEV)
    need = B.lora_cache_chosen_workspace(pool.cache, H, len(q), max(new), budget)
    room = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device=DEV)
    d_ptr = torch.from_numpy(offsets(new)).to(DEV) if ptr == "given" else None
    B.lora_cache_attention_chosen(pool.cache, dtype, H, len(q), max(new), d_ptr, qd, width, out, width, scale, budget, chosen, room if need else None, need)
    torch.cuda.synchronize()
    assert (out[-1] == -7.0).all() and (pad == 0 or (out[:, H * D:] == -7.0).all())
    return out[:-1, :H * D].float().cpu().numpy().reshape(q.shape)


def check_chosen(pool, vals, q, new, lengths, dtype, scale, chosen, got):
    at, G, D, chosen = offsets(new), q.shape[1] // pool.Hkv, q.shape[2], chosen.cpu().numpy()
    for s, n in enumerate(new):
        k, v = (held(x) for x in vals[s])
        _, ks, kz = quantised(vals[s][0])
        _, vs, vz = quantised(vals[s][1])
        for i in range(n):
            row, sees = at[s] + i, max(0, lengths[s] - n + i + 1)
            for g in range(pool.Hkv):
                m = -(-sees // pool.page)
                keep = [x for p in chosen[row, g] if 0 <= p < m and pool.there(s, p * pool.page) for x in range(p * pool.page, min(sees, (p + 1) * pool.page))]
                heads = slice(g * G, (g + 1) * G)
                part = q[row:row + 1, heads]
                if not keep:
                    assert (got[row, heads] == 0).all(), (s, i, g)
                    continue
                # (as in test_attention.py: sums run over codes of up to 31 steps; weights meet codes of at most 7.5 from their middle)
                size = (np.abs(kz[keep, g]) + 31 * ks[keep, g]).max()
                o, tol, amount, _ = reference(part, k[keep][:, g:g + 1], v[keep][:, g:g + 1], scale, lambda _: len(keep), lambda _, h: float(np.abs(part[0, h]).sum() * size))
                tol += (len(keep) / 8 + 64) * 2.0 ** -23 * (np.abs(vz[keep, g]) + 31 * vs[keep, g]).max()
                for h in range(G):
                    x = k[keep, g].astype(np.float64) @ part[0, h].astype(np.float64) * scale
                    e = np.exp(x - x.max())
                    amount[0, h] = (e / e.sum()) @ (7.5 * vs[keep, g])
                check(got[row:row + 1, heads], o, tol, amount, dtype, f"sequence {s}, token {i}, kv head {g}, {len(keep)} slots")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 128), (8, 2, 64), (5, 1, 80), (4, 2, 256), (24, 1, 33), (20, 1, 128), (40, 1, 256)])
@pytest.mark.parametrize("page", [32, 96])
def test_attention_over_chosen_pages(dtype, H, Hkv, D, page):
    """Choices by bounds, and the caller's own: in any order, with numbers that are no pages among them"""
    rng = np.random.default_rng(D + page)
    lengths, new = [1, 0, 33, 700, 300, 2], [1, 0, 4, 3, 1, 4]
    pool = Pool(lengths, Hkv, D, page, seed=H, missing=((4, 1), (3, 2)))
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    bounds, steps = digest(pool, lengths)
    q = rounded(rng.standard_normal((sum(new), H, D)), dtype)
    scale = D ** -0.5
    chosen = run_choose(pool, q, new, dtype, bounds, steps, 4, 1, 1)
    check_chosen(pool, vals, q, new, lengths, dtype, scale, chosen, run_chosen(pool, q, new, dtype, scale, chosen))
    own = np.stack([np.stack([rng.permutation(np.r_[-1:24, -2 ** 31, 2 ** 31 - 1, 700])[:9] for _ in range(Hkv)]) for _ in range(sum(new))]).astype(np.int32)
    own = torch.from_numpy(own).to(DEV)
    check_chosen(pool, vals, q, new, lengths, dtype, scale, own, run_chosen(pool, q, new, dtype, scale, own, pad=3, shift=1))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv", [(8, 2), (32, 1)])
def test_all_pages_chosen_give_what_the_whole_cache_gives(dtype, H, Hkv):
    from test_attention import run_cache
    rng, D = np.random.default_rng(5), 128
    lengths = [1000, 1, 450]
    pool = Pool(lengths, Hkv, D, 64, seed=3, weight=False)
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    bounds, steps = digest(pool, lengths)
    q = rounded(rng.standard_normal((3, H, D)), dtype)
    chosen = run_choose(pool, q, [1, 1, 1], dtype, bounds, steps, 16, 1, 1, ptr=None)
    assert chosen[0].tolist() == [list(range(16))] * Hkv
    got, whole = run_chosen(pool, q, [1, 1, 1], dtype, 0.1, chosen, ptr=None), run_cache(pool, q, [1, 1, 1], dtype, 0.1, ptr=None)
    check_chosen(pool, vals, q, [1, 1, 1], lengths, dtype, 0.1, chosen, got)
    assert np.abs(got - whole).max() <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -18) * np.abs(whole).max()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,budget", [(1, 1, 60), (8, 1, 64), (20, 2, 70)])
def test_many_pages_are_split_and_joined(dtype, H, Hkv, budget):
    rng, D = np.random.default_rng(H), 64
    lengths, new = [5000, 90], [2, 2]
    pool = Pool(lengths, Hkv, D, 64, seed=1)
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    q = rounded(2 * rng.standard_normal((4, H, D)), dtype)
    assert B.lora_cache_chosen_workspace(pool.cache, H, 4, 2, budget) > 0
    chosen = torch.from_numpy(np.stack([[rng.permutation(79)[:budget] if budget < 79 else np.arange(budget) for _ in range(Hkv)] for _ in range(4)]).astype(np.int32)).to(DEV)
    got = run_chosen(pool, q, new, dtype, 0.125, chosen)
    check_chosen(pool, vals, q, new, lengths, dtype, 0.125, chosen, got)
    assert np.array_equal(run_chosen(pool, q, new, dtype, 0.125, chosen), got)
    none = torch.full_like(chosen, -1)
    assert (run_chosen(pool, q, new, dtype, 0.125, none) == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_is_not_chosen_has_no_effect(dtype):
    """NaN and infinities in other pages, in slots behind the token, in what a page holds behind the sequence's end"""
    rng, D, lengths = np.random.default_rng(6), 128, [400, 77]
    pool = Pool(lengths, 1, D, 32, seed=2)
    vals = tokens(rng, lengths, 1, D, dtype)
    pool.fill(vals, dtype)
    q = rounded(rng.standard_normal((4, 4, D)), dtype)
    chosen = torch.tensor([[[3, 12, 0, -1]], [[12, 1, 2, 5]], [[2, 0, -1, -1]], [[2, 1, 0, -1]]], dtype=torch.int32, device=DEV)
    clean = run_chosen(pool, q, [2, 2], dtype, 0.1, chosen)
    check_chosen(pool, vals, q, [2, 2], lengths, dtype, 0.1, chosen, clean)
    for bad in (np.nan, np.inf):
        for s, slots in ((0, range(4 * 32, 5 * 32)), (0, [399]), (1, [76])):
            for x in vals[s]:
                for i in slots:
                    x[i, 0, 5] = bad
        pool.fill(vals, dtype)
        got = run_chosen(pool, q, [2, 2], dtype, 0.1, chosen)
        assert np.array_equal(got[[0, 2]], clean[[0, 2]]) and np.isnan(got[[1, 3]]).all()


@gpu
def test_a_cache_beyond_4_gb():
    page, D, heads = 64, 128, 8
    size = B.lora_cache_page_bytes(page, D)
    n = (1 << 32) // (heads * 2 * D) + 40                    # bounds of more than 4 GB, the cache far beyond
    L = 6 * page - 3
    rng = np.random.default_rng(7)
    pages = torch.empty((n, heads, size), dtype=torch.uint8, device=DEV)
    table = np.array([[n - 1, 3, n - 7, n // 2, n - 20, 1]], np.int32)
    cache = B.lora_cache(pages, torch.from_numpy(table).to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), page, heads, D, L)
    pool = Pool([1], heads, D, page)
    pool.n, pool.table, pool.pages, pool.cache = n, table, pages, cache
    vals = tokens(rng, [L], heads, D, BF16)
    pool.fill(vals, BF16)
    bounds, steps = torch.empty((n, heads, 2, D), dtype=torch.int8, device=DEV), torch.empty((n, heads), device=DEV)
    assert bounds.numel() > 1 << 32
    digest(pool, [L], bounds=bounds, steps=steps)
    q = rounded(rng.standard_normal((1, heads, D)), BF16)
    chosen = run_choose(pool, q, [1], BF16, bounds, steps, 3, 1, 1)
    at = torch.from_numpy(table[0].astype(np.int64)).to(DEV)
    small = Pool([1], heads, D, page)
    small.n, small.table = 6, np.arange(6, dtype=np.int32)[None]
    check_choice(small, q, [1], [L], bounds[at], steps[at], 3, 1, 1, chosen)
    check_chosen(pool, vals, q, [1], [L], BF16, 0.1, chosen, run_chosen(pool, q, [1], BF16, 0.1, chosen))


@gpu
def test_bounds_that_the_call_gives_hold_whatever_the_device_says():
    """Lengths past max_length and below 0, offsets out of order and past the rows, pages of no pool: nothing outside is touched"""
    rng, D = np.random.default_rng(8), 64
    pool = Pool([64, 64, 64], 1, D, 32, max_length=64)
    vals = tokens(rng, [64, 64, 64], 1, D, BF16)
    pool.fill(vals, BF16)
    bounds, steps = digest(pool, [64, 64, 64])
    q = rounded(rng.standard_normal((3, 2, D)), BF16)
    qd = to_device(q, BF16)
    for lengths, ptr in (([2 ** 31 - 1, -5, 64], [0, 1, 2, 3]), ([64, 64, 64], [5, -3, 2 ** 31 - 1, 1]), ([-2 ** 31, 3, 100], [0, 3, 1, 9]), ([64, 64, 64], [2, 1, 0, 0])):
        pool.length.copy_(torch.tensor(lengths, dtype=torch.int32))
        d_ptr = torch.tensor(ptr, dtype=torch.int32, device=DEV)
        b, u = bounds.clone(), steps.clone()
        B.lora_cache_digest(pool.cache, 3, 3, d_ptr, b, u)
        chosen, out = torch.full((4, 1, 2), -9, dtype=torch.int32, device=DEV), torch.full((4, 2 * D), -7.0, dtype=torch.bfloat16, device=DEV)
        B.lora_cache_choose(pool.cache, BF16, 2, 3, 3, d_ptr, qd, 2 * D, b, u, 2, 0, 0, chosen, None, 0)
        need = B.lora_cache_chosen_workspace(pool.cache, 2, 3, 3, 2)
        B.lora_cache_attention_chosen(pool.cache, BF16, 2, 3, 3, d_ptr, qd, 2 * D, out, 2 * D, 0.1, 2, chosen.clamp_min(-9), torch.empty(max(need, 256), dtype=torch.uint8, device=DEV), need)
        torch.cuda.synchronize()
        assert (chosen[3] == -9).all() and (out[3] == -7).all() and ((chosen[:3] >= -1) & (chosen[:3] < 2) | (chosen[:3] == -9)).all()


@gpu
def test_a_captured_decode_step():
    """append, digest, choose, attend as a graph; lengths, tokens and queries change between replays"""
    rng, D, H, Hkv, page = np.random.default_rng(9), 128, 8, 2, 32
    lengths = [300, 40, 7]
    pool = Pool([n + 8 for n in lengths], Hkv, D, page, seed=4, weight=False)
    full = tokens(rng, [n + 8 for n in lengths], Hkv, D, BF16)
    pool.length.copy_(torch.tensor(lengths, dtype=torch.int32))
    pool.fill([[x[:n] for x in v] for v, n in zip(full, lengths)], BF16)
    bounds, steps = digest(pool, lengths)
    k, v, q, out = (torch.zeros((3, h * D), dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, H, H))
    chosen = torch.zeros((3, Hkv, 4), dtype=torch.int32, device=DEV)
    need = B.lora_cache_chosen_workspace(pool.cache, H, 3, 1, 4)
    room = torch.empty(max(256, need), dtype=torch.uint8, device=DEV)

    def step():
        B.lora_cache_append(pool.cache, BF16, 3, 1, None, k, Hkv * D, v, Hkv * D)
        B.lora_cache_digest(pool.cache, 3, 1, None, bounds, steps)
        B.lora_cache_choose(pool.cache, BF16, H, 3, 1, None, q, H * D, bounds, steps, 4, 1, 1, chosen, None, 0)
        B.lora_cache_attention_chosen(pool.cache, BF16, H, 3, 1, None, q, H * D, out, H * D, 0.1, 4, chosen, room, room.numel())
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for i in range(6):
        lengths = [n + 1 for n in lengths]
        pool.length.copy_(torch.tensor(lengths, dtype=torch.int32))
        for x, part in ((k, 0), (v, 1)):
            x.copy_(to_device(np.stack([full[s][part][n - 1] for s, n in enumerate(lengths)]), BF16).view(3, -1))
        values = rounded(rng.standard_normal((3, H, D)), BF16)
        q.copy_(to_device(values, BF16).view(3, -1))
        if i == 0:
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                step()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        graph.replay()
        torch.cuda.synchronize()
        vals = [[x[:n] for x in part] for part, n in zip(full, lengths)]
        whole = digest(pool, lengths)
        rows = torch.from_numpy(np.concatenate([pool.table[s, :-(-n // page)] for s, n in enumerate(lengths)]).astype(np.int64)).to(DEV)
        assert torch.equal(bounds[rows], whole[0][rows]) and torch.equal(steps[rows], whole[1][rows])
        check_choice(pool, values, [1, 1, 1], lengths, bounds, steps, 4, 1, 1, chosen)
        check_chosen(pool, vals, values, [1, 1, 1], lengths, BF16, 0.1, chosen, out.float().cpu().numpy().reshape(3, H, D))


@gpu
def test_a_kv_head_of_many_queries_and_many_tokens():
    rng, D, lengths, new = np.random.default_rng(11), 64, [900, 500], [70, 33]
    pool = Pool(lengths, 1, D, 32, seed=2, weight=False)
    vals = tokens(rng, lengths, 1, D, BF16)
    pool.fill(vals, BF16)
    bounds, steps = digest(pool, lengths)
    q = rounded(rng.standard_normal((sum(new), 18, D)), BF16)
    chosen = run_choose(pool, q, new, BF16, bounds, steps, 3, 0, 1)
    check_choice(pool, q, new, lengths, bounds, steps, 3, 0, 1, chosen)
    check_chosen(pool, vals, q, new, lengths, BF16, 0.125, chosen, run_chosen(pool, q, new, BF16, 0.125, chosen))


# ---- refusals (no GPU) ---------------------------------------------------------------------------------------------------
OK, BAD, UNSUPPORTED, WORKSPACE = B.LORA_OK, B.LORA_ERR_INVALID_ARG, B.LORA_ERR_UNSUPPORTED, B.LORA_ERR_WORKSPACE
MB = 1 << 20
CACHE = dict(pages=64 * MB, weight=None, page_table=1 * MB, length=2 * MB, num_pages=100, num_seqs=4, table_stride=10, max_length=600, page_tokens=64, num_kv_heads=2,
             head_dim=128)


def cache(**f):
    return B.Cache(B.CacheDesc(*[{**CACHE, **f}[n] for n, _ in B.CacheDesc._fields_]))


def status(call):
    try:
        call()
    except B.LoraError as e:
        return e.status
    return OK


DIGEST = dict(num_tokens=4, max_new=1, d_indptr=3 * MB, d_bounds=4 * MB, d_steps=5 * MB)
CHOOSE = dict(dtype=BF16, num_heads=8, num_tokens=4, max_new=1, d_indptr=3 * MB, q=6 * MB, ldq=1024, d_bounds=4 * MB, d_steps=5 * MB, budget=8, first=1, recent=2, d_chosen=7 * MB,
              workspace=None, workspace_bytes=0)
ATTEND = dict(dtype=BF16, num_heads=8, num_tokens=4, max_new=1, d_indptr=3 * MB, q=6 * MB, ldq=1024, o=8 * MB, ldo=1024, scale=0.1, budget=8, d_chosen=7 * MB, workspace=9 * MB,
              workspace_bytes=1 << 30)
CALLS = {"digest": (lambda c, f: B.lora_cache_digest(c, **f, stream=1), DIGEST), "choose": (lambda c, f: B.lora_cache_choose(c, **f, stream=1), CHOOSE),
         "attend": (lambda c, f: B.lora_cache_attention_chosen(c, **f, stream=1), ATTEND)}


def refused(name, c=None, **f):
    call, fine = CALLS[name]
    return status(lambda: call(c or cache(), {**fine, **f}))


@pytest.mark.parametrize("name", list(CALLS))
def test_calls_refuse_what_is_wrong(name):
    for f, expected in ((dict(num_seqs=-1), BAD), (dict(page_tokens=40), BAD), (dict(head_dim=300), BAD), (dict(num_kv_heads=0), BAD), (dict(max_length=641), BAD),
                        (dict(pages=64 * MB + 8), BAD), (dict(pages=None), BAD), (dict(length=None), BAD), (dict(page_table=1 * MB + 2), BAD), (dict(num_pages=1 << 31), UNSUPPORTED)):
        assert refused(name, cache(**f)) == expected, f
    for f in (dict(num_tokens=-1), dict(max_new=-1), dict(d_indptr=3 * MB + 1)):
        assert refused(name, **f) == BAD, f
    assert refused(name, num_tokens=(1 << 30) + 1) == UNSUPPORTED
    for f in (dict(num_tokens=0), dict(max_new=0)):
        assert refused(name, **f) == OK, f
    assert refused(name, cache(num_seqs=0)) == OK


def test_bounds_are_refused():
    for f in (dict(d_bounds=None), dict(d_steps=None), dict(d_bounds=4 * MB + 8), dict(d_steps=5 * MB + 2), dict(d_bounds=64 * MB), dict(d_steps=64 * MB + 64),
              dict(d_steps=4 * MB + 100 * 2 * 256 - 4)):
        assert refused("digest", **f) == BAD, f
        assert refused("choose", **f) == BAD, f
    assert refused("digest", cache(pages=1 << 42, num_seqs=1 << 16, num_kv_heads=1024), d_bounds=1 << 40, d_steps=1 << 41) == UNSUPPORTED


def test_choices_are_refused():
    for f in (dict(dtype=3), dict(num_heads=0), dict(num_heads=3), dict(ldq=1023), dict(q=None), dict(q=6 * MB + 1), dict(budget=0), dict(first=-1), dict(recent=-1),
              dict(first=4, recent=5), dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(d_chosen=None), dict(d_chosen=7 * MB + 2), dict(d_chosen=6 * MB),
              dict(d_chosen=4 * MB), dict(d_chosen=5 * MB), dict(d_chosen=64 * MB)):
        assert refused("choose", **f) == BAD, f
    assert refused("choose", cache(num_seqs=1 << 22, num_kv_heads=2), num_tokens=1 << 22, budget=1, first=0, recent=0) == UNSUPPORTED
    far = cache(page_tokens=32, table_stride=20000, max_length=600000)
    need = B.lora_cache_choose_workspace(far, 4, 1)
    assert need == 4 * 2 * 18752 * 4 // 256 * 256 + 256 * (4 * 2 * 18752 * 4 % 256 > 0) and B.lora_cache_choose_workspace(cache(), 4, 1) == 0
    for f in (dict(workspace=None, workspace_bytes=need), dict(workspace=9 * MB + 16, workspace_bytes=need), dict(workspace=9 * MB, workspace_bytes=need - 1)):
        assert refused("choose", far, **f) == WORKSPACE, f
    for at in (7 * MB, 4 * MB, 5 * MB, 6 * MB, 64 * MB):
        assert refused("choose", far, workspace=at, workspace_bytes=need) == BAD, at


def test_attention_is_refused():
    for f in (dict(dtype=3), dict(num_heads=0), dict(num_heads=3), dict(ldq=1023), dict(ldo=1000), dict(q=None), dict(o=None), dict(q=6 * MB + 1), dict(o=8 * MB + 1), dict(budget=0),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(d_chosen=None), dict(d_chosen=7 * MB + 2), dict(o=6 * MB), dict(o=7 * MB), dict(o=64 * MB)):
        assert refused("attend", **f) == BAD, f
    assert refused("attend", budget=(1 << 24) + 1) == UNSUPPORTED
    assert refused("attend", cache(num_seqs=1 << 22, num_kv_heads=8), num_tokens=1 << 22) == UNSUPPORTED
    c = cache(max_length=640)
    need = B.lora_cache_chosen_workspace(c, 8, 4, 1, 64)
    assert need > 0
    for f in (dict(workspace=None), dict(workspace=9 * MB + 16), dict(workspace_bytes=need - 1)):
        assert refused("attend", c, budget=64, **f) == WORKSPACE, f
    for at in (8 * MB, 7 * MB, 6 * MB, 64 * MB):
        assert refused("attend", c, budget=64, workspace=at) == BAD, at


def test_the_definitions_by_hand():
    k = np.array([[1.0, -2, 0], [0.5, 4, -0.001]], F)
    up, down, step = bounds_of(k)
    assert step == F(4) * THIRD and up.tolist() == [32, 127, 0] and down.tolist() == [15, -64, -1]
    assert codes_of(np.array([2.0, -1, 0], F))[0].tolist() == [127, -64, 0] and codes_of(np.zeros(3, F))[1] == 0 and np.isnan(codes_of(np.array([1, F("inf")]))[1])
    upper, lower = np.array([[1, 0], [0, 0], [5, 0], [5, 0]], np.int8), np.array([[-1, 0], [-9, 0], [0, 0], [0, 0]], np.int8)
    steps = np.ones(4, F)
    assert choice(np.array([[1.0, 0]], F), upper, lower, steps, [True] * 4, 2, 0, 0) == [2, 3]
    assert choice(np.array([[1.0, 0]], F), upper, lower, steps, [True] * 4, 1, 0, 0) == [2]
    assert choice(np.array([[-1.0, 0]], F), upper, lower, steps, [True] * 4, 2, 0, 1) == [1, 3]
    assert choice(np.array([[1.0, 0], [-1, 0]], F), upper, lower, steps, [True, False, True, True], 2, 1, 0) == [0, 2]
