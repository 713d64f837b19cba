"""Attention of prompts, the cache in 4 bits, attention over it and eviction, against the definitions of include/lora_abi.h in 64
bits, and what the calls refuse.

Tolerances, derived: with p the softmax weights and A = sum p |v| / sum p of an output element (64 bits),
    bf16  every p is rounded to 8 bits (2^-8 of it at most) for the product with v, the result once more:  2^-8 (A + |o|)
    all   a score is a 32-bit sum of head_dim products: off by at most head_dim 2^-23 sum |q k| |scale| (+ 2^-22 |score| for its
          scaling and exp2), which changes p by that share, twice (numerator and denominator); sums over n keys in 32 bits: the
          chains are at most n / 8 + 64 long: (n / 8 + 64) 2^-23 A
The cache's products run on codes between 16 and 31 with 23.5 taken off, zero and step apart: the sums' magnitudes are at most 4 times
those of |q| (15 step + |zero|), which is what `sum |q k|` stands for there."""
import ctypes
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B

DEV = "cuda:0"
gpu = pytest.mark.gpu
TORCH = {B.LORA_BF16: torch.bfloat16, B.LORA_F32: torch.float32}
BF16, F32 = B.LORA_BF16, B.LORA_F32


def padded(d):
    return 64 if d <= 64 else 128 if d <= 128 else 256


def rounded(x, dtype):
    t = torch.from_numpy(np.asarray(x, dtype=np.float32))
    return t.to(TORCH[dtype]).float().numpy() if dtype == BF16 else t.numpy()


def to_device(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TORCH[dtype]).to(DEV)


# ---- definitions in 64 bits ----------------------------------------------------------------------------------------------
def reference(q, k, v, scale, sees, products=None):
    """q [n, H, D], k and v [m, Hkv, D]; sees(i): keys [0, sees(i)).  Outputs, their tolerance without the rounding of bf16, A, and
    the weight of every key [m, Hkv].  products: bound of sum |q k| for (query, head) where the keys' own magnitudes are not it."""
    n, H, D = q.shape
    m, G = k.shape[0], H // k.shape[1]
    o, tol, amount, weight = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((m, k.shape[1]))
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for i in range(n):
        c = max(0, min(m, sees(i)))
        for h in range(H):
            if c == 0:
                continue
            kk, vv = k[:c, h // G], v[:c, h // G]
            x = kk @ q[i, h] * scale
            e = np.exp(x - x.max())
            p = e / e.sum()
            o[i, h] = p @ vv
            amount[i, h] = p @ np.abs(vv)
            dot = np.abs(kk) @ np.abs(q[i, h]) if products is None else np.full(c, products(i, h))
            share = (D * 2.0 ** -23 * dot * abs(scale) + 2.0 ** -22 * np.abs(x)).max() + (c / 8 + 64) * 2.0 ** -23
            tol[i, h] = 2 * share * amount[i, h]
            weight[:c, h // G] += p
    return o, tol, amount, weight


def check(got, o, tol, amount, dtype, what=""):
    bound = tol + (2.0 ** -8 * 1.01 * (amount + np.abs(o)) if dtype == BF16 else 2.0 ** -24 * np.abs(o)) + 1e-37
    off = np.abs(got.astype(np.float64) - o)
    assert np.all(off <= bound), f"{what}: {np.max(off / bound):.3g} of the tolerance at {np.unravel_index(np.argmax(off / bound), off.shape)}"


def quantised(x):
    """Codes, steps and zeros of [..., D] (float32 values): the definition, step by step"""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        lo, hi = np.asarray(x.min(-1)), np.asarray(x.max(-1))
        bits = lo.view(np.int32)
        zero = np.where((bits < 0) & (bits & 0xffff != 0), (bits & ~0xffff) + 0x10000, bits & ~0xffff).astype(np.int32).view(np.float32)
        rng = (hi - zero).astype(np.float32)
        step = torch.from_numpy(np.asarray(rng * np.float32(1 / 15), dtype=np.float32)).bfloat16().float().numpy()
        step = np.where(step < 2.0 ** -100, np.float32(0), step)
        bad = ~np.isfinite(x).all(-1) | ~np.isfinite(zero) | ~np.isfinite(rng)
        c = np.clip(np.rint((x - zero[..., None]).astype(np.float32) / np.where(step == 0, 1, step)[..., None].astype(np.float32)), 0, 15)
        c = np.where((step == 0)[..., None] | bad[..., None], 0, c).astype(np.uint8)
    nan = np.float32(np.nan)
    return c, np.where(bad, nan, step).astype(np.float32), np.where(bad, nan, zero).astype(np.float32)


def held(x):
    c, step, zero = quantised(x)
    return c * step[..., None] + zero[..., None]


# ---- prompts -------------------------------------------------------------------------------------------------------------
def prompt_case(rng, nq, nk, H, Hkv, D, dtype, spread=1.0):
    q = rounded(rng.standard_normal((sum(nq), H, D)) * spread, dtype)
    k = rounded(rng.standard_normal((sum(nk), Hkv, D)) + 0.5 * rng.standard_normal((1, Hkv, D)), dtype)
    return q, k, rounded(rng.standard_normal((sum(nk), Hkv, D)) + 0.3, dtype)


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def run_prompt(q, k, v, nq, nk, dtype, causal, scale, pad=0, shift=0, stream=None):
    """pad: elements between rows; shift: of the first element from a 16-byte boundary"""
    def laid(x):
        rows, width = x.shape[0], x.shape[1] * x.shape[2]
        buf = torch.full((rows * (width + pad) + shift + 8,), float("nan"), dtype=TORCH[dtype], device=DEV)
        view = buf[shift:shift + rows * (width + pad)].view(rows, width + pad)
        view[:, :width] = to_device(x, dtype).view(rows, width)
        return view, width + pad
    (qd, ldq), (kd, ldk), (vd, ldv) = laid(q), laid(k), laid(v)
    od, ldo = laid(np.full(q.shape, -7.0))
    plan = B.lora_attention_plan(offsets(nq), offsets(nk), q.shape[1], k.shape[1], q.shape[2], dtype, causal)
    torch.cuda.synchronize()
    B.lora_attention(plan, qd, ldq, kd, ldk, vd, ldv, od, ldo, scale, stream=stream)
    torch.cuda.synchronize()
    if pad:
        assert torch.isnan(od[:, -pad:].float()).all(), "written between the rows"
    plan.destroy()
    return od[:, :q.shape[1] * q.shape[2]].float().cpu().numpy().reshape(q.shape)


def check_prompt(q, k, v, nq, nk, dtype, causal, scale, **layout):
    got = run_prompt(q, k, v, nq, nk, dtype, causal, scale, **layout)
    qo, ko = offsets(nq), offsets(nk)
    for s in range(len(nq)):
        n, m = nq[s], nk[s]
        a, b = slice(qo[s], qo[s + 1]), slice(ko[s], ko[s + 1])
        o, tol, amount, _ = reference(q[a], k[b], v[b], scale, (lambda i: i + m - n + 1) if causal else (lambda i: m))
        check(got[a], o, tol, amount, dtype, f"sequence {s} of {n} queries, {m} keys")
    return got


LENGTHS = [([1], [1]), ([5, 0, 1, 130], [5, 0, 1, 130]), ([64, 65, 31, 33], [64, 65, 31, 33]), ([3, 1, 17], [140, 65, 17]), ([257], [300]),
           ([9, 4, 70], [5, 0, 64])]                        # (the last: queries that see no key, a sequence without one)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", LENGTHS)
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 128), (4, 1, 64), (6, 2, 80), (3, 3, 256)])
def test_prompts(dtype, causal, nq, nk, H, Hkv, D):
    rng = np.random.default_rng(D + len(nq) + nk[0])
    check_prompt(*prompt_case(rng, nq, nk, H, Hkv, D, dtype), nq, nk, dtype, causal, D ** -0.5)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 8, 16, 33, 72, 96, 100, 104, 160, 192, 200])
def test_prompts_of_other_head_dims(dtype, D):
    nq, nk = [70, 3], [75, 3]
    check_prompt(*prompt_case(np.random.default_rng(D), nq, nk, 2, 1, D, dtype), nq, nk, dtype, True, D ** -0.5)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3), (64, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_between_other_columns(dtype, pad, shift, D):
    nq = [40, 100]
    check_prompt(*prompt_case(np.random.default_rng(7), nq, nq, 4, 2, D, dtype), nq, nq, dtype, True, D ** -0.5, pad=pad, shift=shift)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv", [(16, 2), (16, 8), (12, 12), (40, 8), (9, 3), (20, 10), (28, 4)])
def test_prompts_of_many_heads(dtype, H, Hkv):
    """Heads of one kv head in a workgroup of their own or together, runs of them on the XCDs and what is left over"""
    nq, nk = [33, 7, 150, 64], [60, 7, 150, 64]
    check_prompt(*prompt_case(np.random.default_rng(H), nq, nk, H, Hkv, 64, dtype), nq, nk, dtype, True, 0.125)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,pad", [(16, 4, 0), (40, 8, 0), (28, 4, 0), (12, 2, 0), (10, 5, 0), (9, 1, 0), (28, 4, 3)])
def test_many_prompts_of_few_queries(dtype, H, Hkv, pad):
    """Enough of them that a workgroup takes several heads of a tile: 4, 2 and 1 of groups of 4, 5, 7, 6, 2 and 9"""
    rng = np.random.default_rng(H + Hkv)
    nq = rng.integers(0, 34, 70).tolist() + [40, 64, 65]
    nk = [max(0, n + int(rng.integers(-3, 60))) for n in nq]
    plan = B.lora_attention_plan(offsets(nq), offsets(nk), H, Hkv, 64, dtype)
    heads = B.lora_attention_plan_items(plan)[:, 6]
    plan.destroy()
    assert (heads == (2 if H // Hkv == 2 else 4)).any()
    check_prompt(*prompt_case(rng, nq, nk, H, Hkv, 64, dtype), nq, nk, dtype, True, 0.125, pad=pad)


@gpu
def test_prompts_whose_rows_lie_beyond_4_gb():
    nk, D, ld = [20000, 40], 64, 120008
    rng = np.random.default_rng(21)
    nq = [2, 40]
    q, k, v = prompt_case(rng, nq, nk, 2, 1, D, BF16)
    kd, vd = (torch.empty(sum(nk) * ld, dtype=torch.bfloat16, device=DEV).view(sum(nk), ld) for _ in range(2))
    assert kd.numel() * 2 > 1 << 32
    kd[:, :D], vd[:, :D] = to_device(k, BF16).view(-1, D), to_device(v, BF16).view(-1, D)
    qd, od = to_device(q, BF16), torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    plan = B.lora_attention_plan(offsets(nq), offsets(nk), 2, 1, D, BF16)
    B.lora_attention(plan, qd, 2 * D, kd, ld, vd, ld, od, 2 * D, 0.125)
    torch.cuda.synchronize()
    got = od.float().cpu().numpy()
    for a, b, n, m in ((slice(0, 2), slice(0, 20000), 2, 20000), (slice(2, 42), slice(20000, 20040), 40, 40)):
        o, tol, amount, _ = reference(q[a], k[b], v[b], 0.125, lambda i: i + m - n + 1)
        check(got[a], o, tol, amount, BF16)
    plan.destroy()


@gpu
@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("n", [8, 40])
@pytest.mark.parametrize("mb", [17, 31])
def test_few_queries_behind_keys_whose_rows_lie_far_apart(dtype, D, n, mb):
    """A tile's rows beyond 2 GB from its first: what is addressed by 32 bits would come as zeros"""
    m, e = 300, torch.finfo(TORCH[dtype]).bits // 8
    ld = (mb << 20) // e
    q, k, v = prompt_case(np.random.default_rng(mb), [n], [m], 2, 1, D, dtype)
    rows = torch.empty(m * ld, dtype=TORCH[dtype], device=DEV).view(m, ld)            # k and v beside each other
    rows[:, :D], rows[:, D:2 * D] = to_device(k, dtype).view(m, D), to_device(v, dtype).view(m, D)
    qd, od = to_device(q, dtype), torch.zeros(q.shape, dtype=TORCH[dtype], device=DEV)
    plan = B.lora_attention_plan([0, n], [0, m], 2, 1, D, dtype)
    B.lora_attention(plan, qd, 2 * D, rows, ld, rows.data_ptr() + D * e, ld, od, 2 * D, 0.125)
    torch.cuda.synchronize()
    o, tol, amount, _ = reference(q, k, v, 0.125, lambda i: i + m - n + 1)
    check(od.float().cpu().numpy(), o, tol, amount, dtype)
    plan.destroy()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_prompts_with_other_scales(dtype, scale):
    nq, nk = [90, 20], [100, 20]
    check_prompt(*prompt_case(np.random.default_rng(3), nq, nk, 2, 2, 64, dtype), nq, nk, dtype, True, scale)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_whose_scores_grow_along_the_keys(dtype):
    """The running maximum is raised again and again, by little and by much"""
    nq, nk = [130], [700]
    q, k, v = prompt_case(np.random.default_rng(5), nq, nk, 2, 1, 64, dtype)
    k = rounded(k + np.linspace(-6, 6, 700)[:, None, None] * np.sign(q.mean(axis=(0, 1))), dtype)
    check_prompt(q, k, v, nq, nk, dtype, True, 0.125)
    check_prompt(q, k[::-1].copy(), v, nq, nk, dtype, False, 0.125)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("D,shift", [(128, 0), (80, 0), (64, 1)])
@pytest.mark.parametrize("where", ["k", "v", "kv"])
def test_what_a_query_does_not_see_has_no_effect(dtype, bad, D, shift, where):
    """Infinities and NaN in later tokens of the prompt, at its end and in the next sequence"""
    nq, nk = [75, 70, 3], [75, 100, 3]
    q, k, v = prompt_case(np.random.default_rng(11), nq, nk, 4, 2, D, dtype)
    clean = run_prompt(q, k, v, nq, nk, dtype, True, D ** -0.5, shift=shift)
    first = [40, 75 + 80, 175 + 2]                          # rows from which on a sequence holds such values
    kb, vb = k.copy(), v.copy()
    for t in first:
        if "k" in where: kb[t, 1, ::3] = bad
        if "v" in where: vb[t, 1, 1::5] = bad
    got = run_prompt(q, kb, vb, nq, nk, dtype, True, D ** -0.5, shift=shift)
    seen = np.zeros(sum(nq), dtype=bool)
    seen[40:75] = True                                      # (query i of the first sees key i)
    seen[75 + 50:145] = True                                # (of the second: key 80 from query 50 on)
    seen[145 + 2:] = True
    assert np.isfinite(got[~seen]).all()
    if where == "v":                                        # heads of the other kv head: the same bits everywhere
        assert np.array_equal(got[:, :2], clean[:, :2])
    assert np.abs(got[~seen] - clean[~seen]).max() <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -19) * np.abs(clean).max()
    if where != "k" or bad != -np.inf:                      # (a key of -inf elements may just get no weight)
        assert not np.isfinite(got[40:75, 2:]).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,pad", [(64, 0), (40, 0), (80, 0), (128, 0), (136, 0), (256, 0), (128, 3)])
@pytest.mark.parametrize("nq,nk", [([20, 1, 32, 0], [1000, 700, 33, 5]), ([64, 5, 33], [65, 700, 3]), ([3, 7], [129, 0])])
def test_few_queries_behind_many_keys(dtype, causal, D, pad, nq, nk):
    """On a chip that is not full the wavefronts of a workgroup share a tile's keys: four where there are up to 32 queries, two up to 64"""
    check_prompt(*prompt_case(np.random.default_rng(D + len(nq)), nq, nk, 4, 2, D, dtype), nq, nk, dtype, causal, D ** -0.5, pad=pad)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("n", [30, 60])
def test_what_few_queries_do_not_see_has_no_effect(dtype, bad, D, n):
    """Infinities and NaN in values that the last queries see: theirs are not finite, the others' as they were"""
    nq, nk = [n, 9], [300, 200]
    q, k, v = prompt_case(np.random.default_rng(n), nq, nk, 2, 1, D, dtype)
    clean = run_prompt(q, k, v, nq, nk, dtype, True, D ** -0.5)
    vb = v.copy()
    vb[290, 0, 1::5] = bad                                  # seen by the last 10 of the first sequence
    vb[300 + 199, 0, ::7] = bad                             # and by the last of the second
    got = run_prompt(q, k, vb, nq, nk, dtype, True, D ** -0.5)
    seen = np.zeros(sum(nq), dtype=bool)
    seen[n - 10:n] = seen[n + 8] = True
    assert np.isfinite(got[~seen]).all()
    assert np.abs(got[~seen] - clean[~seen]).max() <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -19) * np.abs(clean).max()
    assert not np.isfinite(got[n - 10:n, :, 1::5]).any() and not np.isfinite(got[n + 8, :, ::7]).any()
    others = np.ones(D, dtype=bool)
    others[1::5] = False
    assert np.isfinite(got[n - 10:n][:, :, others]).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [8, 40])
def test_few_queries_whose_scores_grow_or_fall_along_the_keys(dtype, n):
    """The wavefronts' maxima differ by hundreds; one alone has all of the weight"""
    nq, nk, D = [n], [500], 64
    q, k, v = prompt_case(np.random.default_rng(n), nq, nk, 2, 2, D, dtype)
    for slope in (1.0, -1.0):
        q[:, :, 0] = 8.0
        k[:, :, 0] = rounded(slope * np.arange(500)[:, None] / 2 * np.ones((1, 2)), dtype)
        check_prompt(q, k, v, nq, nk, dtype, False, 0.125)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masks_of_the_types_lowest_value_in_keys(dtype):
    """Scores of the type's lowest finite value are scores like others: alone they share the weight"""
    low = float(torch.finfo(TORCH[dtype]).min)
    q = np.zeros((4, 1, 64), np.float32)
    q[:, :, 0] = 1
    k = np.zeros((4, 1, 64), np.float32)
    k[:, :, 0] = low
    v = rounded(np.random.default_rng(1).standard_normal((4, 1, 64)), dtype)
    got = run_prompt(q, k, v, [4], [4], dtype, True, 1.0)
    want = np.stack([v[:i + 1].mean(0) for i in range(4)])
    assert np.abs(got - want).max() <= 2.0 ** -7
    k[3] = 0                                                # ... and beside others they have none
    got = run_prompt(q, k, v, [4], [4], dtype, True, 1.0)
    assert np.array_equal(got[3], v[3])


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, 2e-39, -2e-39, 1e-38])
def test_scales_of_zero_and_below_the_normal_numbers(dtype, scale):
    """Products of up to 1e38 meet them: scores of 0, and of up to 0.2 and 1"""
    rng = np.random.default_rng(4)
    nq, nk = [40], [100]
    q, k, v = prompt_case(rng, nq, nk, 2, 2, 64, dtype)
    q[:], k[:] = 0, 0
    q[:, :, 3] = rounded(1e19, dtype)
    k[:, :, 3] = rounded(1e19 * rng.uniform(-1, 1, (100, 2)), dtype)
    check_prompt(q, k, v, nq, nk, dtype, True, float(np.float32(scale)))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,pad", [(64, 0), (80, 0), (128, 0), (256, 0), (128, 3)])
@pytest.mark.parametrize("nq,nk", [([130, 5], [130, 40]), ([8, 20], [300, 700]), ([50], [600])])
@pytest.mark.parametrize("slope", [0.0, 0.03, -0.03])
def test_values_up_to_the_end_of_their_range(dtype, D, pad, nq, nk, slope):
    """Their mean is in range; the sum of hundreds of them, and one of them times a weight above 1, are not.  slope: the maximum is
    raised by little along the keys, so that weights stay relative to an earlier one"""
    rng = np.random.default_rng(D + nq[0])
    q, k, v = prompt_case(rng, nq, nk, 4, 2, D, dtype)
    q[:, :, 0] = 8.0
    k[:, :, 0] = rounded(slope * np.arange(sum(nk))[:, None] * np.ones((1, 2)), dtype)
    big = 0.9 * float(torch.finfo(TORCH[dtype]).max)
    v = rounded(big * rng.uniform(0.5, 1.0, v.shape) * np.where(rng.random(v.shape) < 0.2, -1, 1), dtype)
    check_prompt(q, k, v, nq, nk, dtype, True, 0.125, pad=pad)


@gpu
def test_prompts_on_a_stream_of_their_own_in_a_graph_and_on_the_current_one():
    nq, D = [130, 40], 128
    q, k, v = (to_device(x, BF16) for x in prompt_case(np.random.default_rng(2), nq, nq, 4, 2, D, BF16))
    plan = B.lora_attention_plan(offsets(nq), None, 4, 2, D, BF16)
    outs = [torch.full_like(q, 7.0) for _ in range(3)]
    side = torch.cuda.Stream()
    B.lora_attention_plan_upload(plan)
    torch.cuda.synchronize()
    call = lambda o, stream=None: B.lora_attention(plan, q, 4 * D, k, 2 * D, v, 2 * D, o, 4 * D, D ** -0.5, stream=stream)
    call(outs[0])
    call(outs[1], side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[2])
    for _ in range(3):
        outs[2].fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[2], outs[0])
    assert torch.equal(outs[1], outs[0])
    plan.destroy()


# ---- the cache -----------------------------------------------------------------------------------------------------------
class Pool:
    """A cache over pages in an order of their own whose memory holds NaN for scales and anything for codes; a page is missing
    where `missing` says so (sequence, page)"""

    def __init__(self, lengths, Hkv, D, page, seed=0, weight=True, spare=1, missing=(), max_length=None):
        rng = np.random.default_rng(seed)
        need = [max(1, -(-n // page)) + spare for n in lengths]
        order = rng.permutation(sum(need) + 2).astype(np.int32)
        self.table = np.full((len(lengths), max(need)), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        for s, p in missing:
            self.table[s, p] = [-1, len(order), 2 ** 31 - 1][(s + p) % 3]
        self.page, self.Hkv, self.D, self.n = page, Hkv, D, len(order)
        size = B.lora_cache_page_bytes(page, D)
        assert size == page * (padded(D) + 8)
        raw = rng.integers(0, 256, (self.n, Hkv, size), dtype=np.uint8)
        raw[..., page * padded(D):] = 0xff                  # words: NaN
        self.pages = torch.from_numpy(raw).to(DEV)
        self.weight = torch.full((self.n, Hkv, page), 3.0, device=DEV) if weight else None
        self.length = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        self.d_table = torch.from_numpy(self.table).to(DEV)
        self.cache = B.lora_cache(self.pages, self.d_table, self.length, page, Hkv, D, max_length or max(max(lengths), 1), self.weight)

    def there(self, s, slot):
        return 0 <= self.table[s, slot // self.page] < self.n

    def fill(self, values, dtype=F32):
        """values: of every sequence, k and v [length, Hkv, D]"""
        k, v = (np.concatenate([x[i] for x in values]) for i in (0, 1))
        ptr = torch.from_numpy(offsets([len(x[0]) for x in values])).to(DEV)
        most = max(len(x[0]) for x in values)
        kd, vd = to_device(k, dtype), to_device(v, dtype)
        ld = self.Hkv * self.D
        B.lora_cache_append(self.cache, dtype, len(k), most, ptr, kd, ld, vd, ld)
        torch.cuda.synchronize()

    def slots(self, tensor, s, n):
        """[n, Hkv] of a per-slot tensor of the pool"""
        out = np.zeros((n, self.Hkv), np.float32)
        x = tensor.cpu().numpy()
        for i in range(n):
            if self.there(s, i):
                out[i] = x[self.table[s, i // self.page], :, i % self.page]
        return out


def tokens(rng, lengths, Hkv, D, dtype):
    return [[rounded(rng.standard_normal((n, Hkv, D)) * np.exp(rng.standard_normal((n, Hkv, 1))) + rng.standard_normal((n, Hkv, 1)), dtype) for _ in range(2)]
            for n in lengths]


def unpacked(pages, page, D):
    """Codes and words of keys and values as the format has them: [pages, Hkv, page, D] and [pages, Hkv, page]"""
    DP = padded(D)
    raw = pages.cpu().numpy()
    N, H = raw.shape[:2]
    half = page * DP // 2
    k = raw[..., :half].reshape(N, H, page, DP // 2)
    v = raw[..., half:2 * half].reshape(N, H, page // 32, 4, 16, 8, DP // 32).transpose(0, 1, 2, 3, 5, 4, 6).reshape(N, H, page, DP // 2)
    words = raw[..., 2 * half:].copy().view(np.uint32).reshape(N, H, 2, page)
    both = [np.stack([x & 15, x >> 4], -1).reshape(N, H, page, DP) for x in (k, v)]
    return both, [words[:, :, 0], words[:, :, 1]]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 7, 40, 64, 80, 100, 128, 200, 256])
@pytest.mark.parametrize("page", [32, 96, 64])
def test_append_holds_the_definitions_codes_and_touches_nothing_else(dtype, D, page):
    rng = np.random.default_rng(D)
    Hkv, before, new = 3, [0, 31, 70, 5], [33, 3, 1, 0]
    lengths = [a + b for a, b in zip(before, new)]
    pool = Pool(lengths, Hkv, D, page, seed=D)
    old = pool.pages.clone()
    vals = tokens(rng, new, Hkv, D, dtype)
    vals[0][0][2, 1] = 1.25                                 # no range: codes 0
    vals[0][0][3, 0, 0] = np.inf
    vals[0][1][4, 2, -1] = np.nan
    vals[0][1][5, 0] = rounded(rng.standard_normal(D) * 1e-32, dtype)
    vals[0][1][6, 0] = rounded(np.linspace(-3.3e38, 3.3e38, D), dtype)
    pool.fill(vals, dtype)
    codes, words = unpacked(pool.pages, page, D)
    touched = np.zeros(words[0].shape, bool)
    for s, n in enumerate(new):
        for i in range(n):
            slot = before[s] + i
            p, at = pool.table[s, slot // page], slot % page
            touched[p, :, at] = True
            for part in range(2):
                c, step, zero = quantised(vals[s][part][i])
                w = words[part][p, :, at]
                bad = np.isnan(step)
                assert np.array_equal(codes[part][p, :, at, :D][~bad], c[~bad])
                assert not codes[part][p, :, at, D:].any()
                assert np.array_equal((w << 16).astype(np.uint32).view(np.float32)[~bad], step[~bad])
                assert np.array_equal((w & 0xffff0000).astype(np.uint32).view(np.float32)[~bad], zero[~bad])
                assert np.isnan((w << 16).astype(np.uint32).view(np.float32)[bad]).all() and np.isnan((w & 0xffff0000).astype(np.uint32).view(np.float32)[bad]).all()
    oc, ow = unpacked(old, page, D)
    for part in range(2):
        assert np.array_equal(words[part][~touched], ow[part][~touched]) and np.array_equal(codes[part][~touched], oc[part][~touched])
    w = pool.weight.cpu().numpy()
    assert (w[touched] == 0).all() and (w[~touched] == 3).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 80, 128, 33, 256])
def test_read_gives_the_values_back(dtype, D):
    rng = np.random.default_rng(D)
    Hkv, lengths = 2, [70, 0, 1, 200]
    pool = Pool(lengths, Hkv, D, 64, missing=[(3, 1)])
    vals = tokens(rng, lengths, Hkv, D, dtype)
    vals[2][0][0, 0, 0] = np.nan
    pool.fill(vals, dtype)
    want = [9, 0, 1, 140]                                   # the last so many of each, one more row in between
    ptr = torch.tensor(offsets(want), dtype=torch.int32, device=DEV)
    k, v = (torch.full((sum(want) + 2, Hkv * D + 5), 9.0, dtype=TORCH[dtype], device=DEV) for _ in range(2))
    B.lora_cache_read(pool.cache, dtype, sum(want) + 2, max(want), ptr, k, Hkv * D + 5, v, Hkv * D + 5)
    torch.cuda.synchronize()
    for part, got in ((0, k), (1, v)):
        got = got.float().cpu().numpy()
        assert (got[:, Hkv * D:] == 9).all() and (got[sum(want):] == 9).all()
        row = 0
        for s, n in enumerate(want):
            for i in range(n):
                slot = lengths[s] - n + i
                expect = rounded(held(vals[s][part][slot]), dtype) if pool.there(s, slot) else np.zeros((Hkv, D), np.float32)
                assert np.array_equal(got[row, :Hkv * D].reshape(Hkv, D), expect, equal_nan=True), (part, s, i)
                row += 1


def run_cache(pool, q, new, dtype, scale, decay=-1.0, ptr="given", pad=0, shift=0):
    H, D = q.shape[1], q.shape[2]
    width = H * D + pad
    buf = torch.zeros(len(q) * width + shift, dtype=TORCH[dtype], device=DEV)
    qd = buf[shift:].view(len(q), width)
    qd[:, :H * D] = to_device(q, dtype).view(len(q), H * D)
    out = torch.full((len(q), width), -7.0, dtype=TORCH[dtype], device=DEV)
    room = B.lora_cache_workspace(pool.cache, H, len(q), max(new), decay >= 0)
    ws = torch.full((max(room, 256),), 0xff, dtype=torch.uint8, device=DEV)          # (NaN: nothing of it may be taken for granted)
    d_ptr = torch.from_numpy(offsets(new)).to(DEV) if ptr == "given" else None
    B.lora_cache_attention(pool.cache, dtype, H, len(q), max(new), d_ptr, qd, width, out, width, scale, decay, ws if room else None, room)
    torch.cuda.synchronize()
    assert pad == 0 or (out[:, H * D:] == -7.0).all()
    return out[:, :H * D].float().cpu().numpy().reshape(q.shape)


def check_cache(pool, vals, q, new, lengths, dtype, scale, got, weight=None):
    """weight: (decay, what was there before) of pool.weight"""
    at = offsets(new)
    D = q.shape[2]
    for s, n in enumerate(new):
        L = lengths[s]
        k, v = (held(x) for x in vals[s])
        there = np.array([pool.there(s, i) for i in range(L)], bool).reshape(-1)
        sees = [max(0, L - n + i + 1) for i in range(n)]
        # magnitude of the sums over codes: |q| times what the zero and 31 steps make of a token
        c, step, zero = quantised(vals[s][0])
        size = (np.abs(zero) + 31 * step)
        G = q.shape[1] // pool.Hkv
        part = q[at[s]:at[s + 1]]
        o, tol, amount, w = (np.zeros(part.shape), np.zeros(part.shape), np.zeros(part.shape), np.zeros((L, pool.Hkv)))
        for i in range(n):
            keep = np.flatnonzero(there[:sees[i]])
            if len(keep) == 0:
                continue
            bound = lambda _, h: float((np.abs(part[i, h]).sum() * size[keep, h // G]).max()) if len(keep) else 0.0
            oo, tt, aa, ww = reference(part[i:i + 1], k[keep], v[keep], scale, lambda _: len(keep), bound)
            # the values' sums run over codes of up to 31 steps, too
            cv, sv, zv = quantised(vals[s][1])
            big = (np.abs(zv[keep]) + 31 * sv[keep]).max(0)
            o[i], tol[i] = oo[0], tt[0] + (len(keep) / 8 + 64) * 2.0 ** -23 * big[np.arange(q.shape[1]) // G][:, None]
            # bf16: rounding p step meets codes of at most 7.5 from their middle, so 2^-8 sum p 7.5 step
            for h in range(q.shape[1]):
                x = k[keep, h // G].astype(np.float64) @ part[i, h].astype(np.float64) * scale
                e = np.exp(x - x.max())
                amount[i, h] = (e / e.sum()) @ (7.5 * sv[keep, h // G])
            w[keep] += ww
        check(got[at[s]:at[s + 1]], o, tol, amount, dtype, f"sequence {s}, {n} tokens on {L}")
        if weight is not None and n:
            decay, before = weight
            expect = decay * before + w
            seen = pool.slots(pool.weight, s, L)
            limit = 2.0 ** -12 * w + 2.0 ** -23 * np.abs(expect) + 1e-30          # of the scores: below, for the inputs here
            assert np.all(np.abs(seen - np.where(there[:, None], expect, 0.0)) <= limit), s


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 128), (8, 2, 64), (5, 1, 80), (4, 2, 256), (3, 3, 33)])
@pytest.mark.parametrize("new", [1, 4, 9])
@pytest.mark.parametrize("page", [32, 64])
def test_attention_over_the_cache(dtype, H, Hkv, D, new, page):
    """Sequences without tokens, shorter than the new tokens (queries that see nothing), ending inside a block and a page"""
    rng = np.random.default_rng(D + new)
    lengths, count = [1, 0, 33, 4, 127, 300], [1, 0, new, new, new, new]
    pool = Pool(lengths, Hkv, D, page, seed=new)
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    before = np.float32(0.75)
    pool.weight.fill_(float(before))
    q = rounded(rng.standard_normal((sum(count), H, D)), dtype)
    scale = D ** -0.5
    got = run_cache(pool, q, count, dtype, scale)
    check_cache(pool, vals, q, count, lengths, dtype, scale, got)
    assert (pool.weight == 0.75).all()
    for decay in (0.0, 0.5, 1.0):
        pool.weight.fill_(float("nan") if decay == 0 else float(before))
        again = run_cache(pool, q, count, dtype, scale, decay)
        assert np.array_equal(again, got, equal_nan=True)
        check_cache(pool, vals, q, count, lengths, dtype, scale, again, (decay, 0.0 if decay == 0 else before))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,new", [(1, 1, 1), (8, 1, 5), (20, 2, 2)])
def test_a_long_cache_is_split_and_joined(dtype, H, Hkv, new):
    rng = np.random.default_rng(H)
    lengths, D = [5000, 40], 64
    pool = Pool(lengths, Hkv, D, 64, seed=1)
    vals = tokens(rng, lengths, Hkv, D, dtype)
    pool.fill(vals, dtype)
    q = rounded(2 * rng.standard_normal((2 * new, H, D)), dtype)
    assert B.lora_cache_workspace(pool.cache, H, 2 * new, new) > 0
    got = run_cache(pool, q, [new, new], dtype, 0.125, 0.0)
    check_cache(pool, vals, q, [new, new], lengths, dtype, 0.125, got, (0.0, 0.0))
    assert np.array_equal(run_cache(pool, q, [new, new], dtype, 0.125, 0.0), got)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_single_tokens_need_no_offsets_and_any_layout_will_do(dtype):
    rng = np.random.default_rng(4)
    lengths, D = [70, 1, 31], 72
    pool = Pool(lengths, 2, D, 32, weight=False)
    vals = tokens(rng, lengths, 2, D, dtype)
    pool.fill(vals, dtype)
    q = rounded(rng.standard_normal((3, 4, D)), dtype)
    got = run_cache(pool, q, [1, 1, 1], dtype, 0.1)
    check_cache(pool, vals, q, [1, 1, 1], lengths, dtype, 0.1, got)
    assert np.array_equal(run_cache(pool, q, [1, 1, 1], dtype, 0.1, ptr=None), got)
    assert np.array_equal(run_cache(pool, q, [1, 1, 1], dtype, 0.1, ptr=None, pad=3, shift=1), got)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [4, 8, 12, 64, 80, 100, 128, 200, 256])
@pytest.mark.parametrize("new", [1, 9])
def test_queries_of_any_alignment_give_the_same(dtype, D, new):
    """16 bytes a lane where rows and heads allow it, element by element elsewhere"""
    rng = np.random.default_rng(D)
    lengths, H = [70, 200, 9], 4
    pool = Pool(lengths, 2, D, 32, weight=False)
    vals = tokens(rng, lengths, 2, D, dtype)
    pool.fill(vals, dtype)
    q = rounded(rng.standard_normal((3 * new, H, D)), dtype)
    got = run_cache(pool, q, [new] * 3, dtype, 0.1)
    check_cache(pool, vals, q, [new] * 3, lengths, dtype, 0.1, got)
    for pad, shift in ((8, 0), (8, 8), (1, 0), (0, 1), (7, 3)):
        assert np.array_equal(run_cache(pool, q, [new] * 3, dtype, 0.1, pad=pad, shift=shift), got), (pad, shift)


@gpu
@pytest.mark.parametrize("decay", [-1.0, 0.0])
def test_more_rows_than_a_tile_and_than_the_weights_take_at_a_time(decay):
    rng = np.random.default_rng(14)
    lengths, new, D = [150, 75], [70, 75], 64
    pool = Pool(lengths, 1, D, 32)
    vals = tokens(rng, lengths, 1, D, BF16)
    pool.fill(vals, BF16)
    q = rounded(rng.standard_normal((145, 4, D)), BF16)
    got = run_cache(pool, q, new, BF16, 0.125, decay)
    check_cache(pool, vals, q, new, lengths, BF16, 0.125, got, None if decay < 0 else (0.0, 0.0))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("lengths,new", [([300, 1, 40], 1), ([300, 33, 40], 9), ([5000], 2), ([2000], 9)])
@pytest.mark.parametrize("v_up,q_up,k_up", [(125, 0, 0), (0, 124, -60), (125, 0, 100), (125, 124, -60)])
def test_values_queries_and_keys_up_to_the_end_of_their_range_in_the_cache(dtype, D, lengths, new, v_up, q_up, k_up):
    """Powers of 2 on the values come out of the mean as they went in, and those on queries and keys go with the scale: what a sum of
    hundreds of codes takes out of range is as near the definition as what none takes out of it.  Elements are below 4, so that 2^125
    times a value is in range and the difference of two is; two results that are within a tolerance each differ by two of them."""
    rng = np.random.default_rng(D + new)
    H, Hkv = 4, 2
    pool = Pool(lengths, Hkv, D, 64)
    few = [min(new, n) for n in lengths]
    vals = [[rounded(np.clip(rng.standard_normal((n, Hkv, D)) + rng.standard_normal((n, Hkv, 1)), -3.5, 3.5), dtype) for _ in range(2)] for n in lengths]
    q = rounded(np.clip(rng.standard_normal((sum(few), H, D)), -3.5, 3.5), dtype)
    pool.fill(vals, dtype)
    base = run_cache(pool, q, few, dtype, D ** -0.5, 0.0).astype(np.float64)
    check_cache(pool, vals, q, few, lengths, dtype, D ** -0.5, base, (0.0, 0.0))
    weights = [pool.slots(pool.weight, s, n) for s, n in enumerate(lengths)]
    pool.fill([[k * np.float32(2.0) ** k_up, v * np.float32(2.0) ** v_up] for k, v in vals], dtype)
    scale = D ** -0.5 * 2.0 ** -(q_up + k_up)
    got = run_cache(pool, q * np.float32(2.0) ** q_up, few, dtype, scale, 0.0).astype(np.float64)
    assert np.isfinite(got).all()
    at = offsets(few)
    for s, n in enumerate(lengths):
        (ck, sk, zk), (cv, sv, zv) = quantised(vals[s][0]), quantised(vals[s][1])
        part = np.abs(q[at[s]:at[s + 1]]).astype(np.float64).sum(-1).max()
        dot = part * (np.abs(zk) + 31 * sk).max() * D ** -0.5
        share = D * 2.0 ** -23 * dot + (n / 8 + 64) * 2.0 ** -23
        most = float((np.abs(zv) + 15 * sv).max())
        tol = 2 * (2 * share * most + (n / 8 + 64) * 2.0 ** -23 * float((np.abs(zv) + 31 * sv).max()))
        if dtype == BF16:
            tol += 2 * 1.01 * 2.0 ** -8 * (7.5 * float(sv.max()) + np.abs(base[at[s]:at[s + 1]]))
        assert np.all(np.abs(got[at[s]:at[s + 1]] * 2.0 ** -v_up - base[at[s]:at[s + 1]]) <= tol), s
        now = pool.slots(pool.weight, s, n)
        assert np.all(np.abs(now - weights[s]) <= 4 * share * weights[s] + 1e-30), s


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,new", [(2, 1), (8, 5)])
@pytest.mark.parametrize("where", [slice(0, 200), slice(2500, 2530), slice(4990, 5000)])
def test_large_values_in_one_piece_of_a_long_cache(dtype, H, new, where):
    """... whose sums are taken smaller, beside pieces whose are not"""
    rng = np.random.default_rng(where.start + new)
    lengths, D = [5000, 40], 64
    pool = Pool(lengths, 1, D, 64)
    vals = tokens(rng, lengths, 1, D, dtype)
    vals[0][1][where] = rounded(np.clip(vals[0][1][where], -3.5, 3.5) * 2.0 ** 120, dtype)
    pool.fill(vals, dtype)
    q = rounded(rng.standard_normal((2 * new, H, D)), dtype)
    got = run_cache(pool, q, [new, new], dtype, 0.125, 0.0)
    assert np.isfinite(got).all()
    check_cache(pool, vals, q, [new, new], lengths, dtype, 0.125, got, (0.0, 0.0))


@gpu
def test_sequences_may_share_the_pages_of_a_prefix():
    """... where no weights are kept: two sequences over the same first 64 tokens, each with its own behind them"""
    rng = np.random.default_rng(31)
    D, lengths, shared = 64, [90, 130], 64
    pool = Pool(lengths, 2, D, 32)
    vals = tokens(rng, lengths, 2, D, BF16)
    for part in range(2):
        vals[1][part][:shared] = vals[0][part][:shared]
    pool.table[1, :2] = pool.table[0, :2]
    pool.d_table.copy_(torch.from_numpy(pool.table))
    for s, new in ((0, 90), (1, 130 - shared)):             # (the prefix is written once)
        kd, vd = (to_device(x[-new:], BF16) for x in vals[s])
        ptr = torch.tensor([0, 0 if s else new, new], dtype=torch.int32, device=DEV)
        B.lora_cache_append(pool.cache, BF16, new, new, ptr, kd, 2 * D, vd, 2 * D)
    q = rounded(rng.standard_normal((4, 4, D)), BF16)
    got = run_cache(pool, q, [2, 2], BF16, 0.125)
    check_cache(pool, vals, q, [2, 2], lengths, BF16, 0.125, got)
    assert np.array_equal(run_cache(pool, q, [2, 2], BF16, 0.125), got)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths", [[4, 100], [5000]])
@pytest.mark.parametrize("score", [1e4, -1e6, 1e6, 1e8, -1e8])
def test_equal_scores_of_any_size_share_the_weight(dtype, lengths, score):
    """In one piece and in several.  Equal scores lie 0 from their maximum, so a row's sum is the count of its keys, exactly, and a
    slot's weight is off by the rounding of 1 / count for each of its rows and of their sum: (rows + 2) 2^-23 of it at most."""
    H, D, new = 8, 64, 2
    pool = Pool(lengths, 1, D, 64)
    vals = [[np.ones((n, 1, D), np.float32), rounded(np.random.default_rng(n).standard_normal((n, 1, D)), dtype)] for n in lengths]
    pool.fill(vals, dtype)
    q = rounded(np.full((new * len(lengths), H, D), score / D), dtype)
    run_cache(pool, q, [new] * len(lengths), dtype, 1.0, 0.0)
    for s, n in enumerate(lengths):
        want = np.full((n, 1), H / n + H / (n - 1))
        want[-1] = H / n                                    # (the first of the two tokens does not see the last slot)
        assert np.all(np.abs(pool.slots(pool.weight, s, n) / want - 1) <= (new * H + 2) * 2.0 ** -23), s


@gpu
def test_a_cache_beyond_4_gb():
    """Pages at the far end of a large pool, tables of int32 page numbers into it"""
    page, Hkv, D, H = 1024, 16, 128, 16
    size = B.lora_cache_page_bytes(page, D)
    count = (5 << 30) // (size * Hkv)
    pages = torch.empty((count, Hkv, size), dtype=torch.uint8, device=DEV)
    assert pages.numel() > 1 << 32
    lengths = [1500, 20]
    table = torch.tensor([[count - 1, 0], [count - 2, 1]], dtype=torch.int32, device=DEV)
    length = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    weight = torch.zeros((count, Hkv, page), device=DEV)
    cache = B.lora_cache(pages, table, length, page, Hkv, D, 2000, weight)
    rng = np.random.default_rng(3)
    vals = tokens(rng, lengths, Hkv, D, BF16)
    kd, vd = (to_device(np.concatenate([x[i] for x in vals]), BF16) for i in (0, 1))
    ptr = torch.tensor(offsets(lengths), device=DEV)
    B.lora_cache_append(cache, BF16, sum(lengths), 1500, ptr, kd, Hkv * D, vd, Hkv * D)
    ko, vo = torch.zeros_like(kd), torch.zeros_like(vd)
    B.lora_cache_read(cache, BF16, sum(lengths), 1500, ptr, ko, Hkv * D, vo, Hkv * D)
    q = to_device(rng.standard_normal((2, H, D)), BF16)
    o = torch.zeros_like(q)
    room = B.lora_cache_workspace(cache, H, 2, 1, True)
    ws = torch.empty(max(room, 256), dtype=torch.uint8, device=DEV)
    B.lora_cache_attention(cache, BF16, H, 2, 1, None, q, H * D, o, H * D, D ** -0.5, 0.0, ws, room)
    torch.cuda.synchronize()
    first = 0
    for s, n in enumerate(lengths):
        for part, got in ((0, ko), (1, vo)):
            assert np.array_equal(got[first:first + n].float().cpu().numpy().reshape(n, Hkv, D), rounded(held(vals[s][part]), BF16))
        first += n
        p = np.zeros((n, Hkv))
        for h in range(H):
            x = held(vals[s][0])[:, h].astype(np.float64) @ q[s, h].double().cpu().numpy() * D ** -0.5
            e = np.exp(x - x.max())
            p[:, h] = e / e.sum()
            want = p[:, h] @ held(vals[s][1])[:, h]
            assert np.linalg.norm(o[s, h].double().cpu().numpy() - want) <= 2.0 ** -6 * np.linalg.norm(want)
        got = np.concatenate([weight[int(table[s, i])].cpu().numpy().T[:max(0, min(page, n - i * page))] for i in range(2)])
        assert np.abs(got - p).max() <= 1e-4


@gpu
def test_bounds_that_the_call_gives_hold_whatever_the_device_says():
    """Lengths past max_length are cut, tokens past max_new and rows past num_tokens left out"""
    rng = np.random.default_rng(15)
    D, Hkv, H = 64, 2, 4
    pool = Pool([100, 60], Hkv, D, 32, max_length=90)
    vals = tokens(rng, [90, 60], Hkv, D, BF16)
    pool.length.copy_(torch.tensor([1000, 60], dtype=torch.int32))          # (90 of the first)
    pool.fill(vals, BF16)
    ptr = torch.tensor([0, 6, 9], dtype=torch.int32, device=DEV)
    q = to_device(rng.standard_normal((9, H, D)), BF16)
    out = torch.full_like(q, 7.0)
    room = B.lora_cache_workspace(pool.cache, H, 8, 4, False)
    ws = torch.empty(max(room, 256), dtype=torch.uint8, device=DEV)
    B.lora_cache_attention(pool.cache, BF16, H, 8, 4, ptr, q, H * D, out, H * D, 0.125, -1.0, ws, room)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy()
    assert (got[4:6] == 7).all() and (got[8:] == 7).all()
    qf = q.float().cpu().numpy()
    for s, rows, last in ((0, range(0, 4), 90 - 6), (1, range(6, 8), 60 - 2)):              # (of the second, two rows are in the call)
        for i, row in enumerate(rows):
            for h in range(H):
                k, v = (held(x)[:last + i + 1, h // 2].astype(np.float64) for x in vals[s])
                x = k @ qf[row, h] * 0.125
                e = np.exp(x - x.max())
                want = (e / e.sum()) @ v
                assert np.linalg.norm(got[row, h] - want) <= 2.0 ** -6 * np.linalg.norm(want), (s, i, h)


@gpu
def test_pages_that_are_not_there_are_not_seen():
    rng = np.random.default_rng(6)
    lengths, D = [200, 130, 40], 64
    pool = Pool(lengths, 2, D, 32, missing=[(0, 2), (0, 6), (1, 0), (2, 0), (2, 1)])      # (of the last, nothing is left)
    vals = tokens(rng, lengths, 2, D, BF16)
    pool.fill(vals, BF16)
    q = rounded(rng.standard_normal((6, 4, D)), BF16)
    got = run_cache(pool, q, [2, 2, 2], BF16, 0.125, 0.0)
    check_cache(pool, vals, q, [2, 2, 2], lengths, BF16, 0.125, got, (0.0, 0.0))
    assert (got[4:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nan_in_the_cache_reaches_the_queries_that_see_it(dtype):
    rng = np.random.default_rng(8)
    lengths, D = [4000, 70], 64
    vals = tokens(rng, lengths, 2, D, dtype)
    vals[0][0][3998, 1, 5] = np.nan                         # seen by the last two of the three tokens, kv head 1
    vals[1][1][69, 0, 2] = np.inf                           # by the last one, kv head 0
    pool = Pool(lengths, 2, D, 64)
    pool.fill(vals, dtype)
    q = rounded(rng.standard_normal((6, 4, D)), dtype)
    got = run_cache(pool, q, [3, 3], dtype, 0.125, 0.0)
    bad = np.zeros((6, 4), bool)
    bad[1:3, 2:] = True
    bad[5, :2] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()


@gpu
def test_lengths_are_read_when_a_graph_is_replayed():
    rng = np.random.default_rng(9)
    D, H = 128, 4
    lengths = [90, 1000]
    vals = tokens(rng, lengths, 2, D, BF16)
    pool = Pool(lengths, 2, D, 64, max_length=1000)
    pool.fill(vals, BF16)
    q = to_device(rng.standard_normal((2, H, D)), BF16)
    room = B.lora_cache_workspace(pool.cache, H, 2, 1, True)
    ws, out = torch.empty(max(room, 256), dtype=torch.uint8, device=DEV), torch.zeros_like(q)
    call = lambda: B.lora_cache_attention(pool.cache, BF16, H, 2, 1, None, q, H * D, out, H * D, D ** -0.5, 0.0, ws, room)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now in ([90, 1000], [17, 333], [0, 64], [90, 1000]):
        pool.length.copy_(torch.tensor(now, dtype=torch.int32))
        pool.weight.zero_()
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got, w = out.clone(), pool.weight.clone()
        pool.weight.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(w, pool.weight), now
        check_cache(pool, [[x[:n] for x in a] for a, n in zip(vals, now)], q.float().cpu().numpy(), [1, 1], now, BF16, D ** -0.5, got.float().cpu().numpy())


# ---- eviction ------------------------------------------------------------------------------------------------------------
def kept_slots(w, length, budget, recent):
    if length <= budget:
        return list(range(length))
    old = length - recent
    x = np.where(np.isnan(w[:old]), np.inf, w[:old])
    order = sorted(range(old), key=lambda i: (not np.isnan(w[i]), -x[i], i))
    return sorted(order[:budget - recent]) + list(range(old, length))


@gpu
@pytest.mark.parametrize("D,page", [(64, 32), (128, 64), (80, 64), (256, 32)])
@pytest.mark.parametrize("budget,recent", [(100, 30), (100, 0), (64, 64), (1, 0), (0, 0), (3000, 10)])
def test_eviction(D, page, budget, recent):
    rng = np.random.default_rng(D + budget)
    Hkv, lengths = 2, [0, 1, 100, 101, 1500, 2500]
    vals = tokens(rng, lengths, Hkv, D, BF16)
    pool = Pool(lengths, Hkv, D, page)
    pool.fill(vals, BF16)
    w = []
    for s, n in enumerate(lengths):
        x = np.round(np.exp(2 * rng.standard_normal((n, Hkv))) * 8).astype(np.float32) / 8       # many ties, zeros among them
        if n > 1000:
            x[7, 0], x[8, 0], x[900, 1], x[11, 1] = np.nan, np.inf, -0.0, -1.5
            x[5, 1] = np.float32(np.uint32(0xffc00001).view(np.float32))                          # (a NaN with its sign set)
        w.append(x)
        flat = pool.weight.cpu().numpy()
        for i in range(n):
            flat[pool.table[s, i // page], :, i % page] = x[i]
        pool.weight.copy_(torch.from_numpy(flat))
    target = Pool([budget] * len(lengths), Hkv, D, page, seed=99, max_length=max(budget, 1))
    source_pages, source_weight = pool.pages.clone(), pool.weight.clone()
    target_pages, target_weight = target.pages.clone(), target.weight.clone()
    kept = torch.full((len(lengths), Hkv, budget), -9, dtype=torch.int32, device=DEV)
    B.lora_cache_evict(pool.cache, target.cache, budget, recent, kept)
    torch.cuda.synchronize()
    assert torch.equal(pool.pages, source_pages) and torch.equal(torch.nan_to_num(pool.weight, 77.0), torch.nan_to_num(source_weight, 77.0))
    assert pool.length.tolist() == lengths and target.length.tolist() == [min(n, budget) for n in lengths]
    kept = kept.cpu().numpy()
    (sk, sv), (skw, svw) = unpacked(pool.pages, page, D)
    (tk, tv), (tkw, tvw) = unpacked(target.pages, page, D)
    touched = np.zeros(tkw.shape, bool)
    tw = target.weight.cpu().numpy()
    for s, n in enumerate(lengths):
        for h in range(Hkv):
            want = kept_slots(w[s][:, h], n, budget, recent)
            assert kept[s, h].tolist() == want + [-1] * (budget - len(want)), (s, h)
            for j, i in enumerate(want):
                a, b = (pool.table[s, i // page], h, i % page), (target.table[s, j // page], h, j % page)
                touched[b] = True
                assert np.array_equal(tk[b], sk[a]) and np.array_equal(tv[b], sv[a]) and tkw[b] == skw[a] and tvw[b] == svw[a]
                assert np.array_equal(tw[b], w[s][i, h], equal_nan=True)
    (ok, ov), (okw, ovw) = unpacked(target_pages, page, D)
    assert np.array_equal(tkw[~touched], okw[~touched]) and np.array_equal(tk[~touched], ok[~touched]) and np.array_equal(tv[~touched], ov[~touched])
    assert np.array_equal(tvw[~touched], ovw[~touched]) and np.array_equal(tw[~touched], target_weight.cpu().numpy()[~touched])


@gpu
@pytest.mark.parametrize("length,budget,recent", [(4096, 1000, 0), (4500, 4097, 3), (5000, 700, 100), (32768, 9000, 0), (40000, 1234, 34), (40000, 39990, 1)])
def test_eviction_of_long_caches(length, budget, recent):
    rng = np.random.default_rng(length + budget)
    Hkv, D, page = 2, 64, 128
    pool = Pool([length, 17], Hkv, D, page)
    w = np.exp(3 * rng.standard_normal((length, Hkv))).astype(np.float32)
    w[rng.random(w.shape) < 0.3] = 0                        # exactly none
    w[:, 1] = np.round(w[:, 1])                             # ties everywhere
    flat = pool.weight.cpu().numpy()
    i = np.arange(length)
    flat[pool.table[0, i // page], :, i % page] = w
    pool.weight.copy_(torch.from_numpy(flat))
    target = Pool([budget, budget], Hkv, D, page, seed=3)
    kept = torch.full((2, Hkv, budget), -9, dtype=torch.int32, device=DEV)
    B.lora_cache_evict(pool.cache, target.cache, budget, recent, kept)
    torch.cuda.synchronize()
    for h in range(Hkv):
        want = kept_slots(w[:, h], length, budget, recent)
        assert kept[0, h].tolist() == want
        assert kept[1, h].tolist() == (list(range(17)) + [-1] * budget)[:budget]
        a, b = pool.table[0, np.array(want) // page], np.array(want) % page
        c, d = target.table[0, np.arange(budget) // page], np.arange(budget) % page
        assert np.array_equal(target.weight.cpu().numpy()[c, h, d], w[want, h])
        (sk, sv), (skw, svw) = unpacked(pool.pages, page, D)
        (tk, tv), (tkw, tvw) = unpacked(target.pages, page, D)
        assert np.array_equal(tk[c, h, d], sk[a, h, b]) and np.array_equal(tv[c, h, d], sv[a, h, b])
        assert np.array_equal(tkw[c, h, d], skw[a, h, b]) and np.array_equal(tvw[c, h, d], svw[a, h, b])


@gpu
def test_a_cache_lives_through_prompt_decode_and_eviction():
    """Attention over what eviction left equals attention over the kept tokens, new ones appended behind them"""
    rng = np.random.default_rng(12)
    lengths, D, H, Hkv, budget = [500, 90], 64, 4, 2, 200
    vals = tokens(rng, lengths, Hkv, D, BF16)
    pool = Pool(lengths, Hkv, D, 64)
    pool.fill(vals, BF16)
    q = rounded(2 * rng.standard_normal((16, H, D)), BF16)
    run_cache(pool, q, [8, 8], BF16, 0.125, 0.0)
    w = [pool.slots(pool.weight, s, n) for s, n in enumerate(lengths)]
    target = Pool([budget] * 2, Hkv, D, 64, seed=5, max_length=budget + 64)
    kept = torch.empty((2, Hkv, budget), dtype=torch.int32, device=DEV)
    B.lora_cache_evict(pool.cache, target.cache, budget, 32, kept)
    torch.cuda.synchronize()
    now = []
    for s, n in enumerate(lengths):
        want = [kept_slots(w[s][:, h], n, budget, 32) for h in range(Hkv)]
        assert [kept[s, h, :len(want[h])].tolist() for h in range(Hkv)] == want
        now.append([np.stack([x[want[h], h] for h in range(Hkv)], 1) for x in vals[s]])
    fresh = tokens(rng, [3, 2], Hkv, D, BF16)
    target.length += torch.tensor([3, 2], dtype=torch.int32, device=DEV)
    ptr = torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV)
    kd, vd = (to_device(np.concatenate([f[i] for f in fresh]), BF16) for i in (0, 1))
    B.lora_cache_append(target.cache, BF16, 5, 3, ptr, kd, Hkv * D, vd, Hkv * D)
    vals = [[np.concatenate([a, b]) for a, b in zip(x, f)] for x, f in zip(now, fresh)]
    q = rounded(rng.standard_normal((5, H, D)), BF16)
    got = run_cache(target, q, [3, 2], BF16, 0.125)
    check_cache(target, vals, q, [3, 2], [203, 92], BF16, 0.125, got)


# ---- plans and calls (no GPU) --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 4), (8, 1), (32, 8), (40, 40), (28, 4), (9, 3), (12, 2), (64, 8)])
@pytest.mark.parametrize("causal", [True, False])
def test_a_plans_items_cover_every_query_of_every_head_once(H, Hkv, causal):
    rng = np.random.default_rng(H)
    for nq, nk in LENGTHS + [(rng.integers(0, 700, 40).tolist(), rng.integers(0, 900, 40).tolist()), ([], []), ([0, 0], [5, 0])]:
        plan = B.lora_attention_plan(offsets(nq), offsets(nk), H, Hkv, 64, BF16, causal)
        items = B.lora_attention_plan_items(plan)
        seen = np.zeros((sum(nq), H), int)
        qo, ko = offsets(nq), offsets(nk)
        assert len(items) % 8 == 0
        for row, rows, key, keys, ahead, most, heads, head in items:
            if heads == 0:
                continue
            s = int(np.searchsorted(qo, row, side="right")) - 1
            assert qo[s] <= row and row + rows <= qo[s + 1] and (key, keys) == (ko[s], nk[s]) and 1 <= rows <= 128
            first = row - qo[s]
            sees = [max(0, min(nk[s], nk[s] - nq[s] + first + i + 1)) if causal else nk[s] for i in range(rows)]
            assert [max(0, min(keys, ahead + i + 1)) for i in range(rows)] == sees and most == sees[-1]
            assert heads in (1, 2, 4) and head // (H // Hkv) == (head + heads - 1) // (H // Hkv) and heads * rows <= 128
            seen[row:row + rows, head:head + heads] += 1
        assert (seen == 1).all()
        # the XCDs' shares (every eighth item): none has more than its part and the heaviest unit of heads
        load = [sum(int(i[5]) + 64 for i in items[x::8] if i[6]) for x in range(8)]
        unit = max((int(i[5]) + 64 for i in items if i[6]), default=0) * 4 * max(1, -(-len(items) // max(H, 1)))
        assert max(load) - min(load) <= unit
        plan.destroy()


@pytest.mark.parametrize("group,runs", [(1, [1]), (2, [2]), (3, [2, 1]), (4, [4]), (5, [4, 1]), (6, [4, 2]), (7, [4, 2, 1]), (8, [4, 4]), (9, [4, 4, 1])])
def test_heads_of_few_queries_go_together(group, runs):
    plan = B.lora_attention_plan(np.arange(401) * 20, None, 2 * group, 2, 64, BF16)
    items = B.lora_attention_plan_items(plan)
    items = items[items[:, 6] > 0]
    for kv in (0, 1):
        first = items[(items[:, 0] == 0) & (items[:, 7] // group == kv)]
        assert first[np.argsort(first[:, 7]), 6].tolist() == runs
    plan.destroy()
    plan = B.lora_attention_plan([0, 20], None, 2 * group, 2, 64, BF16)       # a chip that is not full: one by one
    items = B.lora_attention_plan_items(plan)
    assert set(items[items[:, 6] > 0, 6]) == {1}
    plan.destroy()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 64, 80, 96, 100, 128, 200, 256])
@pytest.mark.parametrize("n,shared", [(8, 4), (40, 2), (128, 1)])
def test_all_rows_of_a_tile_lie_where_its_loads_reach(dtype, D, n, shared):
    """Loads straight to LDS reach 2^31 bytes; a tile whose rows lie further apart is made smaller or goes through registers"""
    plan = B.lora_attention_plan([0, n], [0, 300 + n], 2, 1, D, dtype)
    for pitch in (1024, 2 ** 24 - 16, 2 ** 24, 17 << 20, 31 << 20, 2 ** 25 - 16, 2 ** 25, 2 ** 26 - 16, 2 ** 26, 2 ** 33, 2 ** 40):
        dims, keys, sharing, direct = B.lora_attention_plan_instance(plan, True, pitch)
        assert dims >= D and (not direct or keys * pitch < 2 ** 31)
        assert direct == (pitch < 2 ** 26 if keys == 32 else pitch < 2 ** 25)
        assert sharing in (1, shared, 2 if dtype == F32 else shared)
        assert B.lora_attention_plan_instance(plan, False, pitch)[2:] == (1, False)
    assert B.lora_attention_plan_instance(plan, True, 1024)[2] == (1 if D > 128 else 2 if dtype == F32 and D > 64 and n <= 64 else shared)
    plan.destroy()


def test_plans_are_the_same_for_the_same_batch():
    a, b = (B.lora_attention_plan(offsets([5, 300, 70]), None, 12, 4, 80, F32) for _ in range(2))
    assert np.array_equal(B.lora_attention_plan_items(a), B.lora_attention_plan_items(b))


P, I32, I64, F, Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
ABI = {"lora_attention_plan_upload": [P, P], "lora_attention": [P, P, I64, P, I64, P, I64, P, I64, F, P],
       "lora_cache_append": [P, I32, I32, I32, P, P, I64, P, I64, P], "lora_cache_read": [P, I32, I32, I32, P, P, I64, P, I64, P],
       "lora_cache_attention": [P, I32, I32, I32, I32, P, P, I64, P, I64, F, F, P, Z, P], "lora_cache_evict": [P, P, I32, I32, P, P]}


@pytest.mark.parametrize("calls", ["_calls", "calls_ctypes"])
@pytest.mark.parametrize("name", list(ABI))
def test_arguments_reach_the_abi(calls, name):
    """By position and by name, in place; what is missing or too much is refused"""
    import importlib
    import inspect
    import types
    module = importlib.import_module("paper_2411_00915_amd." + calls)
    seen, status = [], [0]
    keep = [ctypes.CFUNCTYPE(ctypes.c_int, *arguments)(lambda *a, n=n: (seen.append((n, list(a))), status[0])[1]) for n, arguments in ABI.items()]
    if calls == "calls_ctypes":
        module.bind(B._check, B._first_stream, *[B._address(keep[0])] * 8)
    module.bind_attention(*(B._address(f) for f in keep))
    try:
        function = getattr(module, name)
        parameters = inspect.signature(function).parameters
        assert list(parameters) == list(inspect.signature(getattr(B, name)).parameters)
        values = {p: types.SimpleNamespace(handle=0x1000 + i) if p in ("plan", "cache", "target") else 0.25 if p in ("scale", "decay") else 64 + i
                  for i, p in enumerate(parameters)}
        expected = [0x1000 + i if p in ("plan", "cache", "target") else v for i, (p, v) in enumerate(values.items())]
        function(*values.values())
        function(**dict(reversed(values.items())))
        assert seen == [(name, expected)] * 2
        for wrong in (list(values.values())[:-2], [*values.values(), 0]):
            with pytest.raises(TypeError):
                function(*wrong)
        status[0] = B.LORA_ERR_WORKSPACE
        with pytest.raises(B.LoraError, match=f"{name}: workspace"):
            function(**values)
    finally:
        if calls == "_calls":
            module.bind_attention(*(B._address(getattr(B._lib, n)) for n in ABI))


# ---- refusals (no GPU) ---------------------------------------------------------------------------------------------------
def test_the_definitions_by_hand():
    c, step, zero = quantised(np.array([-1.0, 0.0, 14.0, 2.0], np.float32))
    assert step == 1.0 and zero == -1.0 and c.tolist() == [0, 1, 15, 3]
    c, step, zero = quantised(np.array([2.0, 2.0], np.float32))
    assert step == 0.0 and zero == 2.0 and c.tolist() == [0, 0]
    c, step, zero = quantised(np.array([-1.001, 0.0], np.float32))                    # down to bf16: -1.0078125
    assert zero == -1.0078125 and abs(step - 1.0078125 / 15) <= 2.0 ** -8 * step
    assert np.isnan(held(np.array([1.0, np.inf], np.float32))).all()
    assert kept_slots(np.array([1, 5, 5, 0, 2, 9], np.float32), 6, 3, 1) == [1, 2, 5]
    assert kept_slots(np.array([np.nan, 5, np.inf, 0], np.float32), 4, 1, 0) == [0]


def test_attention_plans_refuse_what_is_wrong():
    ok = dict(q=[0, 3, 3, 10], k=[0, 5, 5, 5], H=4, Hkv=2, D=64, dtype=BF16, causal=1)

    def status(**f):
        f = {**ok, **f}
        q, k = (None if x is None else np.asarray(x, np.int32) for x in (f["q"], f["k"]))
        ptr = lambda x: None if x is None else x.ctypes.data_as(B._i32p)
        desc = B.AttentionDesc(f.get("S", 3), ptr(q), ptr(k), f["H"], f["Hkv"], f["D"], f["dtype"], f["causal"])
        st, handle = B.lora_attention_plan_create_raw(desc)
        assert (handle is None) == (st != B.LORA_OK)
        if handle:
            B.AttentionPlan(handle).destroy()
        return st

    assert status() == B.LORA_OK and status(k=None) == B.LORA_OK and status(D=1) == B.LORA_OK and status(D=256) == B.LORA_OK
    assert status(q=[0], k=None, S=0) == B.LORA_OK
    for wrong in (dict(q=None), dict(q=[1, 3, 3, 10]), dict(q=[0, 3, 2, 10]), dict(k=[0, 5, 4, 5]), dict(k=[2, 5, 5, 5]), dict(S=-1), dict(H=0), dict(Hkv=0),
                  dict(H=5), dict(D=0), dict(D=257), dict(dtype=2), dict(causal=2), dict(causal=-1)):
        assert status(**wrong) == B.LORA_ERR_INVALID_ARG, wrong
    assert status(q=[0, 0, 0, 2 ** 30 + 1]) == B.LORA_ERR_UNSUPPORTED and status(k=[0, 0, 0, 2 ** 31 - 1]) == B.LORA_ERR_UNSUPPORTED
    assert B.lora_attention_plan_create_raw(None)[0] == B.LORA_ERR_INVALID_ARG
    assert B._lib.lora_attention_plan_create(None, None) == B.LORA_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        B.lora_attention_plan([0, 3], [0, 3, 4], 1, 1, 64, BF16)


def test_attention_refuses_what_is_wrong():
    plan = B.lora_attention_plan([0, 3], None, 4, 2, 64, BF16)
    ok = dict(q=4096, ldq=256, k=8192, ldk=128, v=4096 * 3, ldv=128, o=4096 * 4, ldo=256, scale=1.0)
    for wrong in (dict(q=0), dict(k=0), dict(v=0), dict(o=0), dict(ldq=255), dict(ldk=127), dict(ldv=127), dict(ldo=255), dict(q=4097), dict(k=4097),
                  dict(v=4097), dict(o=4097), dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(B.LoraError, match="lora_attention") as e:
            B.lora_attention(plan, **{**ok, **wrong}, stream=0)
        assert e.value.status == B.LORA_ERR_INVALID_ARG, wrong
    with pytest.raises(B.LoraError):
        B.lora_attention(B.AttentionPlan(None), **ok, stream=0)
    empty = B.lora_attention_plan([0, 0], [0, 7], 4, 2, 64, BF16)
    B.lora_attention(empty, **{**ok, "q": 0, "o": 0}, stream=0)                       # nothing to do
    with pytest.raises(B.LoraError):
        B.lora_attention_plan_upload(B.AttentionPlan(None), stream=0)


def fake(**f):
    """A descriptor over addresses that no call may touch"""
    d = dict(pages=1 << 20, weight=1 << 21, page_table=1 << 22, length=1 << 23, num_pages=8, num_seqs=2, table_stride=4, max_length=200, page_tokens=64,
             num_kv_heads=2, head_dim=64)
    d.update(f)
    return B.Cache(B.CacheDesc(*(d[n] for n, _ in B.CacheDesc._fields_)))


WRONG_CACHES = [dict(pages=None), dict(pages=(1 << 20) + 8), dict(page_table=None), dict(length=None), dict(num_pages=-1), dict(num_seqs=-1),
                dict(table_stride=-1), dict(max_length=-1), dict(max_length=257), dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=1056),
                dict(page_tokens=-64), dict(num_kv_heads=0), dict(head_dim=0), dict(head_dim=257), dict(page_table=(1 << 22) + 2), dict(weight=(1 << 21) + 1)]


def test_the_caches_calls_refuse_what_is_wrong():
    calls = {"append": lambda c, dtype=BF16, n=2, most=1, k=4096, ldk=128, v=8192, ldv=128: B.lora_cache_append(c, dtype, n, most, None, k, ldk, v, ldv, stream=0),
             "read": lambda c, dtype=BF16, n=2, most=1, k=4096, ldk=128, v=8192, ldv=128: B.lora_cache_read(c, dtype, n, most, None, k, ldk, v, ldv, stream=0),
             "attention": lambda c, dtype=BF16, n=2, most=1, H=4, q=4096, ldq=256, o=8192, ldo=256, scale=1.0, decay=-1.0, ws=1 << 24, size=1 << 30:
                 B.lora_cache_attention(c, dtype, H, n, most, None, q, ldq, o, ldo, scale, decay, ws, size, stream=0)}

    def refused(name, c, status=B.LORA_ERR_INVALID_ARG, **f):
        with pytest.raises(B.LoraError, match=f"lora_cache_{name}") as e:
            calls[name](c, **f)
        assert e.value.status == status, (name, f)

    for name in calls:
        for wrong in WRONG_CACHES:
            refused(name, fake(**wrong))
        refused(name, fake(), dtype=2)
        refused(name, fake(), n=-1)
        refused(name, fake(), most=-1)
        refused(name, B.Plan(None, None))
        calls[name](fake(), n=0)                            # nothing to do
        calls[name](fake(), most=0)
        calls[name](fake(num_seqs=0, pages=None), n=4)
        refused(name, fake(num_pages=1 << 31), status=B.LORA_ERR_UNSUPPORTED)
        refused(name, fake(), status=B.LORA_ERR_UNSUPPORTED, n=2 ** 30 + 1)
    for name in ("append", "read"):
        for f in (dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=127), dict(k=4097), dict(v=4097), dict(dtype=F32, k=4098)):
            refused(name, fake(), **f)
    for f in (dict(q=None), dict(o=None), dict(ldq=255), dict(ldo=255), dict(q=4097), dict(o=4097), dict(H=0), dict(H=5), dict(scale=float("nan")),
              dict(decay=float("nan")), dict(decay=1.5)):
        refused("attention", fake(), **f)
    refused("attention", fake(weight=None), decay=0.5)
    need = B.lora_cache_workspace(fake(), 4, 2, 1, True)
    assert need > 0
    refused("attention", fake(), status=B.LORA_ERR_WORKSPACE, decay=0.5, size=need - 1)
    refused("attention", fake(), status=B.LORA_ERR_WORKSPACE, decay=0.5, ws=None)
    refused("attention", fake(), status=B.LORA_ERR_WORKSPACE, decay=0.5, ws=(1 << 24) + 64)
    with pytest.raises(B.LoraError):
        B.lora_cache_workspace(fake(), 5, 2, 1)
    assert B._lib.lora_cache_workspace(fake().handle, 4, 2, 1, 0, None) == B.LORA_ERR_INVALID_ARG
    assert B.lora_cache_workspace(fake(), 4, 0, 1) == 0

    for f in (dict(n=2 ** 29, H=8), dict(n=2 ** 20, most=2 ** 31 - 1, H=4)):                # rows past 32 bits, of all and of all sequences
        refused("attention", fake(num_seqs=2 ** 12), status=B.LORA_ERR_UNSUPPORTED, **f)
    with pytest.raises(B.LoraError):                        # a workspace of a few TB
        B.lora_cache_workspace(fake(max_length=2 ** 30, table_stride=2 ** 24), 1024, 2 ** 10, 1, True)
    assert B.lora_cache_workspace(fake(), 4, 2, 2 ** 31 - 1, True) == B.lora_cache_workspace(fake(), 4, 2, 2, True)

    def evict_refused(source, target, budget=100, recent=10, kept=4096, status=B.LORA_ERR_INVALID_ARG):
        with pytest.raises(B.LoraError, match="lora_cache_evict") as e:
            B.lora_cache_evict(source, target, budget, recent, kept, stream=0)
        assert e.value.status == status

    other = dict(length=1 << 25)
    for wrong in WRONG_CACHES:
        evict_refused(fake(**wrong), fake(**other))
        evict_refused(fake(), fake(**{**other, **wrong}))
    for wrong in (dict(num_seqs=3), dict(num_kv_heads=1), dict(head_dim=128), dict(page_tokens=128), dict(max_length=99), dict(weight=None)):
        evict_refused(fake(), fake(**{**other, **wrong}))
    evict_refused(fake(weight=None), fake(**other))
    evict_refused(fake(), fake())                           # one array of lengths for both
    for f in (dict(budget=-1), dict(recent=-1), dict(recent=101), dict(kept=None), dict(kept=4097)):
        evict_refused(fake(), fake(**other), **f)
    evict_refused(B.Plan(None, None), fake(**other))


def test_caches_of_more_than_2_to_30_tokens_are_refused():
    """(slots and the ends of splits are 32-bit numbers)"""
    for length, status in ((2 ** 30 + 1, B.LORA_ERR_UNSUPPORTED), (2 ** 31 - 1, B.LORA_ERR_UNSUPPORTED)):
        long = fake(max_length=length, table_stride=2 ** 25)
        for call in (lambda: B.lora_cache_append(long, BF16, 2, 1, None, 4096, 128, 8192, 128, stream=0),
                     lambda: B.lora_cache_read(long, BF16, 2, 1, None, 4096, 128, 8192, 128, stream=0),
                     lambda: B.lora_cache_attention(long, BF16, 4, 2, 1, None, 4096, 256, 8192, 256, 1.0, -1.0, 1 << 24, 1 << 40, stream=0),
                     lambda: B.lora_cache_workspace(long, 4, 2, 1),
                     lambda: B.lora_cache_evict(long, fake(length=1 << 25), 100, 10, 4096, stream=0)):
            with pytest.raises(B.LoraError) as e:
                call()
            assert e.value.status == status
    assert B.lora_cache_workspace(fake(max_length=2 ** 30, table_stride=2 ** 24), 4, 2, 1) > 0


def test_launches_of_too_many_threads_are_refused():
    """2^24 workgroups of 256 threads are more than a launch holds"""
    seqs = np.arange(2 ** 14 + 1, dtype=np.int32)
    for heads, fits in ((8, True), (1024, False)):
        desc = B.AttentionDesc(2 ** 14, seqs.ctypes.data_as(B._i32p), None, heads, heads, 64, BF16, 1)
        st, handle = B.lora_attention_plan_create_raw(desc)
        assert st == (B.LORA_OK if fits else B.LORA_ERR_UNSUPPORTED)
        if handle:
            B.AttentionPlan(handle).destroy()
    many = fake(num_kv_heads=2 ** 20, num_seqs=2 ** 4)
    for call in (lambda: B.lora_cache_append(many, BF16, 1024, 64, 4096, 4096, 2 ** 26, 8192, 2 ** 26, stream=0),
                 lambda: B.lora_cache_read(many, BF16, 1024, 64, 4096, 4096, 2 ** 26, 8192, 2 ** 26, stream=0),
                 lambda: B.lora_cache_attention(many, BF16, 2 ** 20, 16, 1, None, 4096, 2 ** 26, 8192, 2 ** 26, 1.0, -1.0, 1 << 24, 1 << 40, stream=0),
                 lambda: B.lora_cache_workspace(many, 2 ** 20, 16, 1),
                 lambda: B.lora_cache_evict(many, fake(num_kv_heads=2 ** 20, num_seqs=2 ** 4, length=1 << 25), 100, 10, 4096, stream=0)):
        with pytest.raises(B.LoraError) as e:
            call()
        assert e.value.status == B.LORA_ERR_UNSUPPORTED


def test_an_append_of_too_many_threads_is_refused():
    """Its workgroups have 320 threads, not 256: the bound is 2^32 / 320 of them.  (What is refused here does not reach the device.)"""
    most = (2 ** 32 - 1) // 320
    call = lambda f, heads, n: f(fake(num_kv_heads=heads, head_dim=1, num_seqs=2), BF16, n, 64, 4096, 4096, heads, 8192, heads, stream=0)
    for heads in (1, 128, 4096):
        n = (most // heads + 1) * 32                        # one workgroup more than that, for every head
        if n > 2 ** 30:
            n = 2 ** 30 + 1
        with pytest.raises(B.LoraError) as e:
            call(B.lora_cache_append, heads, n)
        assert e.value.status == B.LORA_ERR_UNSUPPORTED, heads
        with pytest.raises(B.LoraError) as e:               # a tile's last token counts as the whole tile
            call(B.lora_cache_append, heads, n - 31)
        assert e.value.status == B.LORA_ERR_UNSUPPORTED, heads


def test_outputs_that_share_memory_with_inputs_are_refused():
    plan = B.lora_attention_plan([0, 3, 10], [0, 3, 20], 4, 2, 64, BF16)               # 10 rows of 512 bytes, 20 of 256
    base = 1 << 20

    def refused(call):
        with pytest.raises(B.LoraError) as e:
            call()
        assert e.value.status == B.LORA_ERR_INVALID_ARG

    far = dict(q=base, ldq=256, k=base << 1, ldk=128, v=base << 2, ldv=128, o=base << 3, ldo=256, scale=1.0)
    for f in (dict(o=base), dict(o=base + 9 * 512 + 510), dict(o=base - 9 * 512 - 510), dict(o=(base << 1) + 19 * 256), dict(o=(base << 2) - 9 * 512),
              dict(o=base, ldo=512, ldq=512), dict(o=base + 512 - 2, ldo=512, ldq=512), dict(o=base + 1024 * 5 + 1024 - 510, ldo=512, ldq=512),      # same pitch
              dict(o=base + 1024 - 510, ldo=512, ldq=512), dict(o=base - 1024 * 3 - 2, ldo=512, ldq=512), dict(o=(base << 1) + 130, ldo=4096, ldk=128),
              dict(o=(base << 1) - 1024 * 9, ldo=512)):                                 # the last row alone meets the keys
        refused(lambda: B.lora_attention(plan, **{**far, **f}, stream=0))
    for k, v in ((base + 73000, 8192), (4096, base), (base - 200, 8192)):             # the pages
        for call in (B.lora_cache_read, B.lora_cache_append):
            refused(lambda: call(fake(), BF16, 2, 1, None, k, 128, v, 128, stream=0))
    refused(lambda: B.lora_cache_read(fake(), BF16, 2, 1, None, (1 << 22) + 100, 128, 1 << 22, 128, stream=0))        # its two outputs
    for q, o in ((4096, 4096), (4096, 4096 + 1022), (4096, base), (base + 200000, base + 199000), (4096, base - 1000)):
        refused(lambda: B.lora_cache_attention(fake(), BF16, 4, 2, 1, None, q, 256, o, 256, 1.0, -1.0, 1 << 24, 1 << 30, stream=0))


@gpu
def test_outputs_may_lie_beside_inputs_in_the_rows_of_one_buffer():
    rng = np.random.default_rng(6)
    n, m, H, Hkv, D = 33, 50, 4, 2, 64
    q, k, v = prompt_case(rng, [n], [m], H, Hkv, D, BF16)
    width = (2 * H + 2 * Hkv) * D
    rows = torch.zeros((m, width), dtype=torch.bfloat16, device=DEV)                   # q, o, k, v: of the last two, more rows
    for x, first in ((q, 0), (k, 2 * H * D), (v, (2 * H + Hkv) * D)):
        rows[:len(x), first:first + x.shape[1] * D] = to_device(x, BF16).view(len(x), -1)
    plan = B.lora_attention_plan([0, n], [0, m], H, Hkv, D, BF16)
    at = lambda first: rows.data_ptr() + 2 * first
    B.lora_attention(plan, at(0), width, at(2 * H * D), width, at((2 * H + Hkv) * D), width, at(H * D), width, 0.125)
    torch.cuda.synchronize()
    o, tol, amount, _ = reference(q, k, v, 0.125, lambda i: i + m - n + 1)
    check(rows[:n, H * D:2 * H * D].float().cpu().numpy().reshape(n, H, D), o, tol, amount, BF16)
    assert (rows[n:, :2 * H * D] == 0).all()
    plan.destroy()
    # ... and one behind the other
    both = torch.zeros((2 * n, H * D), dtype=torch.bfloat16, device=DEV)
    both[:n] = to_device(q, BF16).view(n, -1)
    kd, vd = to_device(k, BF16), to_device(v, BF16)
    plan = B.lora_attention_plan([0, n], [0, m], H, Hkv, D, BF16)
    B.lora_attention(plan, both, H * D, kd, Hkv * D, vd, Hkv * D, both[n:], H * D, 0.125)
    torch.cuda.synchronize()
    assert torch.equal(both[n:], rows[:n, H * D:2 * H * D])
    plan.destroy()


def test_bytes_of_a_page():
    assert [B.lora_cache_page_bytes(64, d) for d in (1, 64, 65, 128, 129, 256)] == [64 * 72, 64 * 72, 64 * 136, 64 * 136, 64 * 264, 64 * 264]
    assert [B.lora_cache_page_bytes(*a) for a in ((0, 64), (31, 64), (33, 64), (1056, 64), (64, 0), (64, 257), (-32, 64))] == [0] * 7


def test_descriptors_are_made_of_fitting_tensors():
    pages, table, length = torch.zeros(4, 2, 64 * 72, dtype=torch.uint8), torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = B.lora_cache(pages, table, length, 64, 2, 64, 100)
    assert (c.desc.num_pages, c.desc.num_seqs, c.desc.table_stride, c.desc.max_length, c.desc.weight) == (4, 3, 5, 100, None)
    for bad in (dict(pages=pages.float()), dict(page_table=table.long()), dict(length=length[:2]), dict(pages=pages.flatten()[:-1]), dict(page_tokens=33),
                dict(weight=torch.zeros(4, 2, 63)), dict(page_table=table.t()), dict(length=length.double())):
        f = dict(pages=pages, page_table=table, length=length, page_tokens=64, num_kv_heads=2, head_dim=64, max_length=100)
        with pytest.raises(ValueError):
            B.lora_cache(**{**f, **bad})


def test_the_descriptors_have_the_headers_layout(tmp_path):
    """Offsets of the fields as a C compiler sees them"""
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"lora_cache": B.CacheDesc, "lora_attention_desc": B.AttentionDesc}
    lines = [f'printf("%zu ", sizeof({n}));' + "".join(f'printf("%zu ", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in structs.items()]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "lora_abi.h"\nint main(void) {' + "".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I" + os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    assert out == [x for s in structs.values() for x in [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
