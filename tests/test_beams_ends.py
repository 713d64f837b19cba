"""Beam selection where its sums are at an end of what they can be, against the definition in 64 bits as in test_beams.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B
from test_beams import BF16, DEV, F32, TORCH, check, gpu, run, scores


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,some", [(4096, 4096), (5000, 5000), (9001, 4000), (70000, 40000), (300, 300)])
@pytest.mark.parametrize("out", [3, 64])
@pytest.mark.parametrize("groups", [1, 60])
def test_many_logits_of_the_largest_finite_number(dtype, vocab, some, out, groups):
    """More than LDS holds candidates, with nothing above them that could be a bound; also beside what is lower, below it by a step, and -inf.
    A row's log sum is the largest number + log(some), which in 64 bits is that number: all are worth the row's score"""
    rng, beams, top = np.random.default_rng(some), 3, float(torch.finfo(TORCH[dtype]).max)
    x = np.full((groups * beams, vocab), top, np.float64)
    for r, low in zip(range(len(x)), (1.0, -np.inf, top * (1 - torch.finfo(TORCH[dtype]).eps), -top)):
        x[r, rng.permutation(vocab)[: vocab - some]] = low
    check(x.astype(np.float32), scores(rng, len(x)), None, 0, beams, out, dtype)


@gpu
@pytest.mark.parametrize("dtype,groups,beams,vocab,out", [(BF16, 64, 8, 131072, 16), (F32, 64, 4, 50021, 4), (BF16, 200, 4, 60000, 8), (F32, 300, 4, 20001, 64), (BF16, 2, 4, 32000, 8)])
def test_the_same_bits_again(dtype, groups, beams, vocab, out):
    """Rows of several units a workgroup: scores, parents and tokens, and the sums that the second launch reads (two numbers of 64 bits for each piece of a row, at
    the workspace's start), call after call, beside other work and on a stream of its own"""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(vocab)
    x = (torch.randn((groups * beams, vocab), generator=gen, device=DEV) * 3).to(TORCH[dtype])
    score = torch.rand(groups * beams, generator=gen, device=DEV) - 9
    need = B.lora_beam_workspace(groups, beams, vocab, out)
    pieces = next(n for n in range(1, 1 << 14) if need == -(-(-(-n * groups * beams * 16 // 256) * 256 + n * groups * beams * out * 8) // 256) * 256)
    others, first = [torch.cuda.Stream(), torch.cuda.Stream()], None
    side = torch.randn((2048, 2048), device=DEV)
    torch.cuda.synchronize()
    for i in range(24):
        got = [torch.empty((groups, out), dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
        room = torch.zeros(need, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        if i % 2:
            with torch.cuda.stream(others[0]):
                side = torch.tanh(side @ side)
        with torch.cuda.stream(others[1] if i % 3 else torch.cuda.current_stream()):
            B.lora_beam_select(dtype, groups, beams, vocab, x, vocab, score, None, 0, out, *got, room, need)
        torch.cuda.synchronize()
        bits = [got[0].view(torch.int32), got[1], got[2], room[: pieces * groups * beams * 16]]
        first = bits if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(first, bits)), i


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [5000, 131072, 1 << 20])
@pytest.mark.parametrize("floor", ["equal", "two", "spread"])
def test_a_peak_over_a_floor(dtype, vocab, floor):
    """One logit above all others, which together weigh as much as it, or far more, or less: the log sum is made of exponentials in 32 bits.

    With u = 2^-24 and g the reference less the logit: the argument g log2(e) is rounded once (u of itself, so g u of the exponential), log2(e) in 32
    bits is 0.224 u of itself off (0.224 g u), exp2 is off by 2 u, and of eight that are added the sum by 7 u.  The weighted mean of g is at most log(vocab): with
    weights w = exp(-g) / Z it is the weights' entropy less log Z, and Z is 1 or more, as the largest logit is not below the reference.  So
    a log sum is off by at most (9 + 1.225 log(vocab)) u; a score of it is rounded once more."""
    rng = np.random.default_rng(vocab)
    gaps, bases = np.arange(1.0, 17.0, 0.6180339887), np.array([4.0, -9.0, 0.0, 117.0])
    if vocab > 1 << 17:
        gaps = gaps[::4]
    off = []
    for base in bases:
        x = np.full((len(gaps), vocab), base)
        if floor == "two":
            x[:, rng.permutation(vocab)[: vocab // 3]] -= 1.3
        if floor == "spread":
            x -= rng.random((1, vocab)) * 2
        place = rng.integers(0, vocab, len(gaps))
        x[np.arange(len(gaps)), place] = base + gaps
        x = torch.from_numpy(x.astype(np.float32)).to(TORCH[dtype]).float().numpy()
        got, parent, token = run(x, np.zeros(len(gaps), np.float32), None, 0, 1, 2, dtype)
        x = x.astype(np.float64)
        top = x.max(1, keepdims=True)
        expect = x - top - np.log(np.exp(x - top).sum(1, keepdims=True))
        rest = x.copy()
        rest[np.arange(len(gaps)), place] = -np.inf
        second = rest.argmax(1)
        assert (token[:, 0] == place).all() and (token[:, 1] == second).all() and (parent == np.arange(len(gaps))[:, None]).all()
        expect = np.take_along_axis(expect, np.stack([place, second], 1), 1)
        off.append(np.abs(got - expect))
        assert np.all(off[-1] <= (9 + 1.225 * np.log(vocab)) * 2.0 ** -24 + 2.0 ** -24 * np.abs(expect)), (base, off[-1].max())
    print(f"{floor}, {vocab}: greatest difference of the peak's score {max(o[:, 0].max() for o in off):.2e}")
