"""The attention layer of serve_layer.py, from prompts through decode steps and an eviction, against the same in 64 bits.

What the reference shares with the layer are the slots that each eviction kept (weights that lie close together may change
places by a rounding); everything else it computes from the inputs.  Tolerance: values pass five roundings to bf16 (q, k, v;
softmax weights; attention's output; the layer's output), 2^-9 each in the mean, that add up as squares: 2^-9 sqrt(5) = 0.44 %
of the norm; codes of the cache that fall to the other side of a tie because k or v was rounded the other way: one step of 15
in at most one of a thousand, 0.3 %.  Together 0.6 %; the test asks for 1.5 %."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_attention import held

pytestmark = pytest.mark.gpu


def project(p, x, adapters):
    """x [tokens, k] in 64 bits, adapters of the tokens"""
    y = x @ p.Wt.double().cpu().numpy().T
    for i, a in enumerate(adapters):
        if a >= 0:
            y[i] += float(p.scale[a]) * (x[i] @ p.At[a].double().cpu().numpy().T) @ p.Bt[a].double().cpu().numpy().T
    return y


def bf16(x):
    return torch.from_numpy(np.asarray(x)).bfloat16().double().numpy()


def softmax_sum(q, k, v):
    s = k @ q / np.sqrt(len(q))
    p = np.exp(s - s.max())
    return (p / p.sum()) @ v, p / p.sum()


def test_prompts_decode_steps_and_eviction():
    from paper_2411_00915_amd.serve_layer import AttentionLayer, DEV
    S, H, Hkv, D, hidden, limit, budget, recent = 4, 4, 2, 64, 256, 72, 40, 8
    layer = AttentionLayer(hidden, H, Hkv, D, [8, 16, 24], S, limit, budget, recent, page=32, window=8)
    rng = np.random.default_rng(1)
    lengths, adapters = [70, 1, 33, 50], [0, -1, 2, 1]
    of = np.repeat(adapters, lengths)
    x = bf16(rng.standard_normal((sum(lengths), hidden)))
    got = layer.prompts(torch.from_numpy(x).bfloat16().to(DEV), lengths, adapters).double().cpu().numpy()
    split = lambda y: (y[:, :H * D].reshape(-1, H, D), y[:, H * D:(H + Hkv) * D].reshape(-1, Hkv, D), y[:, (H + Hkv) * D:].reshape(-1, Hkv, D))
    q, k, v = split(bf16(project(layer.qkv, x, of)))
    o, cache, first = np.zeros((len(x), H * D)), [], 0
    for n in lengths:
        for i in range(first, first + n):
            for h in range(H):
                o[i, h * D:(h + 1) * D] = softmax_sum(q[i, h], k[first:i + 1, h * Hkv // H], v[first:i + 1, h * Hkv // H])[0]
        cache.append([[held(m[first:first + n, g].astype(np.float32)).astype(np.float64) for g in range(Hkv)] for m in (k, v)])
        first += n
    near = lambda a, b, what: print(what, np.linalg.norm(a - b) / np.linalg.norm(b)) or np.linalg.norm(a - b) <= 0.015 * np.linalg.norm(b)
    assert near(got, project(layer.out, bf16(o), of), "prompts")
    evictions = 0
    evict = layer.evict

    def watched():
        nonlocal evictions
        evictions += 1
        before = list(layer.lengths)
        kept = evict().cpu().numpy()
        for s in range(S):
            for g in range(Hkv):
                slots = kept[s, g][kept[s, g] >= 0]
                assert len(slots) == min(budget, before[s]) and (np.diff(slots) > 0).all()
                assert before[s] <= budget or slots[-recent:].tolist() == list(range(before[s] - recent, before[s]))
                for part in range(2):
                    cache[s][part][g] = cache[s][part][g][slots]
    layer.evict = watched
    for step in range(40):
        x = bf16(rng.standard_normal((S, hidden)))
        got = layer.decode(torch.from_numpy(x).bfloat16().to(DEV), adapters).double().cpu().numpy()
        q, k, v = split(bf16(project(layer.qkv, x, adapters)))
        o = np.zeros((S, H * D))
        for s in range(S):
            for g in range(Hkv):
                for part, m in ((0, k), (1, v)):
                    cache[s][part][g] = np.concatenate([cache[s][part][g], held(m[s, g].astype(np.float32))[None].astype(np.float64)])
            for h in range(H):
                o[s, h * D:(h + 1) * D] = softmax_sum(q[s, h], cache[s][0][h * Hkv // H], cache[s][1][h * Hkv // H])[0]
        assert near(got, project(layer.out, bf16(o), adapters), f"step {step}")
        assert layer.lengths == layer.cache.length.tolist() == [len(c[0][0]) for c in cache]
    assert evictions == 2


def test_plans_of_past_batches_are_given_back():
    from paper_2411_00915_amd.serve_layer import DEV, Projection
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    p = Projection(256, 256, [8, 16, 24], 2.0, gen)
    x = torch.randn((9, 256), generator=gen, device=DEV).bfloat16()
    batches = [([n, 9 - n], [n % 3, (n + 1) % 3]) for n in range(10)] + [([4, 5], [2, 0]), ([9], [1])]
    first = [p(x, *b) for b in batches]
    assert len(p.plans) == Projection.KEPT == len({plan.handle for plan, _ in p.plans.values()})
    held = list(p.plans.values())
    for b, y in zip(batches, first):
        assert torch.equal(p(x, *b), y)
    assert len(p.plans) == Projection.KEPT and list(p.plans)[-1] == ((9,), (1,))
    assert any(not plan.handle for plan, _ in held)             # (destroyed)
    p(x, *batches[-3])                                          # one that is held: it is now the last to go
    assert list(p.plans)[-1] == tuple(map(tuple, batches[-3])) and len(p.plans) == Projection.KEPT


def test_the_command_runs():
    from paper_2411_00915_amd import serve_layer
    assert serve_layer.main(["--requests", "3", "--prompt", "40", "--steps", "12", "--hidden", "256", "--heads", "4", "--kv-heads", "2", "--limit", "64",
                             "--budget", "48"]) == 0
