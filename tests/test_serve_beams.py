"""Beam search over the serving layer of serve_layer.py: prompts, then steps in which beams share pages, part and end, against the same in 64 bits.

What the reference shares with the layer are the beams that each selection took (candidates that lie close together may change places by a
rounding of the logits), which is checked against the layer's own logits, and, where pages are chosen, the pages.
Tolerance of the logits: values pass five roundings to bf16 up to the layer's output (test_serve_layer.py: 0.6 % of the norm with the codes that
fall to the other side of a tie) and one more behind the last product, 2^-9 in the mean: 0.65 %; the test asks for 1.5 %."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_attention import held
from test_beams import NEAR, worth
from test_serve_layer import bf16, project, softmax_sum

pytestmark = pytest.mark.gpu


def near(a, b, what):
    off = np.linalg.norm(a - b) / np.linalg.norm(b)
    assert off <= 0.015, (what, off)


def check_selection(logits, score, last, end, beams, groups, got):
    """Of the layer's own logits the best, in order"""
    s, parent, token = (x.cpu().numpy().reshape(groups, -1) for x in got)
    vocab = logits.shape[1]
    for g in range(groups):
        rows = slice(g * beams, (g + 1) * beams)
        c = worth(logits[rows], score[rows], np.zeros(beams, bool) if last is None or end < 0 else last[rows] == end, end).ravel()
        at = (parent[g] - g * beams) * vocab + token[g]
        best = np.sort(c)[::-1][:len(at)]
        assert len(set(at.tolist())) == len(at) and np.all(np.abs(c[at] - best) <= NEAR) and np.all(np.abs(s[g] - c[at]) <= 2.0 ** -22 + 2.0 ** -24 * np.abs(c[at]))


@pytest.mark.parametrize("chosen", [0, 2])
@pytest.mark.parametrize("K", [1, 3])
def test_beams_from_prompts_on(K, chosen):
    from paper_2411_00915_amd.serve_layer import BeamLayer, DEV
    R, H, Hkv, D, hidden, vocab, page = 3, 4, 2, 64, 256, 1000, 32

    def make(end_token):
        return BeamLayer(hidden, H, Hkv, D, [8, 16, 24], R, K, 128, vocab, page=page, chosen=chosen, end_token=end_token)
    rng = np.random.default_rng(2)
    lengths, adapters = [70, 1, 64], [0, -1, 2]
    x = bf16(rng.standard_normal((sum(lengths), hidden)))
    xd = torch.from_numpy(x).bfloat16().to(DEV)
    layer = make(-1)
    layer.prompts(xd, lengths, adapters)
    layer.step()
    end = int(layer.token[0])                               # (a token that is taken in the second step: beams end there)
    layer = make(end)
    for again in range(2):                                  # (requests that were there before give their pages back)
        layer.prompts(xd, lengths, adapters)
    split = lambda y: (y[:, :H * D].reshape(-1, H, D), y[:, H * D:(H + Hkv) * D].reshape(-1, Hkv, D), y[:, (H + Hkv) * D:].reshape(-1, Hkv, D))  # noqa: E731
    E = layer.embedding.double().cpu().numpy()
    q, k, v = split(bf16(project(layer.qkv, x, np.repeat(adapters, lengths))))
    o, cache, first = np.zeros((R, H * D)), [], 0
    for r, n in enumerate(lengths):
        for h in range(H):
            g = h * Hkv // H
            o[r, h * D:(h + 1) * D] = softmax_sum(q[first + n - 1, h], k[first:first + n, g], v[first:first + n, g])[0]
        cache.append([held(m[first:first + n].astype(np.float32)).astype(np.float64) for m in (k, v)])
        first += n
    near(layer.logits.double().cpu().numpy(), bf16(project(layer.out, bf16(o), adapters)) @ E.T, "prompts")
    check_selection(layer.logits.float().cpu().numpy(), np.zeros(R, np.float32), None, -1, 1, R, layer.best)
    cache = [cache[p // K] for p in layer.parent.tolist()]
    ended = 0
    for step in range(24):
        token, score = layer.token.cpu().numpy(), layer.score.cpu().numpy()
        ended += int((token == end).sum())
        layer.step()
        assert layer.granted.all()
        xs = E[token]
        q, k, v = split(bf16(project(layer.qkv, xs, np.repeat(adapters, K))))
        o = np.zeros((R * K, H * D))
        for s in range(R * K):
            cache[s] = [np.concatenate([old, held(new[s:s + 1].astype(np.float32)).astype(np.float64)]) for old, new in zip(cache[s], (k, v))]
            n = len(cache[s][0])
            for h in range(H):
                g = h * Hkv // H
                keep = np.arange(n)
                if chosen:
                    pages = [p for p in layer.list[s, g].tolist() if p >= 0]
                    assert len(pages) == min(chosen, -(-n // page)) and pages == sorted(set(pages)) and pages[0] == 0 and pages[-1] == (n - 1) // page
                    keep = np.concatenate([np.arange(p * page, min(n, (p + 1) * page)) for p in pages])
                o[s, h * D:(h + 1) * D] = softmax_sum(q[s, h], cache[s][0][keep, g], cache[s][1][keep, g])[0]
        near(layer.logits.double().cpu().numpy(), bf16(project(layer.out, bf16(o), np.repeat(adapters, K))) @ E.T, f"step {step}")
        check_selection(layer.logits.float().cpu().numpy(), score, token, end, K, R, layer.best)
        cache = [cache[p] for p in layer.parent.tolist()]
        length, table = layer.length.tolist(), layer.table.cpu().numpy()
        assert length == [len(c[0]) for c in cache]
        named = np.concatenate([table[s, :-(-n // page)] for s, n in enumerate(length)])
        assert np.array_equal(np.bincount(named, minlength=len(layer.users)), layer.users.cpu().numpy())
    assert ended > 0


def test_the_command_searches_with_beams():
    from paper_2411_00915_amd import serve_layer
    assert serve_layer.main(["--requests", "3", "--prompt", "40", "--steps", "12", "--hidden", "256", "--heads", "4", "--kv-heads", "2", "--limit", "64",
                             "--budget", "48", "--beams", "3", "--vocab", "500", "--chosen", "2"]) == 0
