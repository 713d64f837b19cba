"""One attention layer of a multi-LoRA serving program, from prompts to decode steps, through the library's calls:

    prompts      lora_fused_forward (q, k and v of every request with its own adapter) -> lora_attention -> lora_cache_append,
                 lora_cache_attention of the last tokens (how much weight every cached token gets) -> lora_fused_forward (output)
    decode step  lora_fused_forward -> lora_cache_append -> lora_cache_attention (weights carried on) -> lora_fused_forward
    eviction     lora_cache_evict, where the caches have grown past their limit, into pages of their own
    beams        lora_pages_resize (pages for the step's tokens) -> lora_cache_copy (of pages that beams shared) -> lora_fused_forward -> lora_cache_append ->
                 lora_cache_attention, or lora_cache_digest, lora_cache_choose and lora_cache_attention_chosen -> lora_fused_forward -> lora_base_gemm (logits) ->
                 lora_beam_select -> lora_pages_fork (every beam becomes its parent)

    python -m paper_2411_00915_amd.serve_layer [--requests 32] [--prompt 512] [--steps 64] [--hidden 4096] [--heads 32]
                                               [--kv-heads 8] [--limit 600] [--budget 512] [--beams 4] [--vocab 32000] [--chosen 0]

prints microseconds per layer of the prompts, of a decode step and of an eviction, and of a step of beam search (chosen: pages that a token attends
to, 0: all).  Random weights; rotary positions, norms and the MLP are the program's own and left out here.
"""
import argparse
import sys
import time

import numpy as np
import torch

from . import binding as B

DEV = "cuda:0"


class Projection:
    """y = x W + s (x A_a) B_a for the requests' adapters: the weight, the factors and their pointer tables, and the plans of the last few
    batches"""
    KEPT = 8                                                    # plans: decode steps take one again and again, every prompt batch one of its own

    def __init__(self, k, n, ranks, scale, gen):
        def randn(*size, std):
            return (torch.randn(size, generator=gen, device=DEV) * std).bfloat16()
        self.k, self.n, self.ranks, self.scale = k, n, np.asarray(ranks, np.int32), np.full(len(ranks), scale, np.float32)
        self.Wt = randn(n, k, std=k ** -0.5)
        self.At = [randn(int(r), k, std=k ** -0.5) for r in ranks]
        self.Bt = [randn(n, int(r), std=float(r) ** -0.5) for r in ranks]
        self.At_ptrs, self.Bt_ptrs = (torch.tensor([m.data_ptr() for m in ms], dtype=torch.int64, device=DEV) for ms in (self.At, self.Bt))
        self.plans = {}

    def __call__(self, x, lengths, adapters):
        """x [tokens, k] of requests of these lengths, each on its adapter"""
        key = (tuple(lengths), tuple(adapters))                # (a program plans once a batch, for all of its layers)
        if key in self.plans:
            self.plans[key] = self.plans.pop(key)              # (the latest used is last)
        else:
            if len(self.plans) >= self.KEPT:
                torch.cuda.synchronize()                       # (a plan is given back when the work that uses it is through)
                self.plans.pop(next(iter(self.plans)))[0].destroy()
            plan = B.lora_plan(sum(lengths), np.concatenate([[0], np.cumsum(lengths)]), adapters, self.ranks, self.scale, self.k, self.n, B.LORA_BF16)
            B.lora_plan_upload(plan)
            room = torch.empty(max(256, B.lora_plan_query(plan)[2]), dtype=torch.uint8, device=DEV)
            self.plans[key] = plan, room
        plan, room = self.plans[key]
        y = torch.empty((x.shape[0], self.n), dtype=torch.bfloat16, device=DEV)
        B.lora_fused_forward(plan, x, self.k, self.Wt, self.k, self.At_ptrs, self.Bt_ptrs, y, self.n, room, room.numel())
        return y


class Pages:
    """Pages of one layer's cache and the free ones among them"""

    def __init__(self, count, page, kv_heads, head_dim):
        self.pages = torch.empty((count, kv_heads, B.lora_cache_page_bytes(page, head_dim)), dtype=torch.uint8, device=DEV)
        self.weight = torch.empty((count, kv_heads, page), device=DEV)
        self.free = list(range(count))[::-1]

    def take(self, count):
        if count > len(self.free):
            raise RuntimeError("no page of the cache is free")
        return [self.free.pop() for _ in range(count)]


class AttentionLayer:
    def __init__(self, hidden, heads, kv_heads, head_dim, ranks, requests, limit, budget, recent, page=64, window=16, scale=2.0, seed=0):
        """limit: tokens of a request's cache at which all caches are brought down to `budget`, the last `recent` ones kept;
        window: the last tokens of a prompt whose attention ranks its tokens"""
        if not 0 <= recent <= budget < limit:
            raise ValueError("0 <= recent <= budget < limit")
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.page, self.window = heads, kv_heads, head_dim, page, window
        self.limit, self.budget, self.recent, self.requests = limit, budget, recent, requests
        self.qkv = Projection(hidden, (heads + 2 * kv_heads) * head_dim, ranks, scale, gen)
        self.out = Projection(heads * head_dim, hidden, ranks, scale, gen)
        each = -(-limit // page)
        self.pool = Pages(2 * requests * each, page, kv_heads, head_dim)             # (the caches, and what an eviction fills)
        self.stride, self.lengths = each, [0] * requests
        self.cache = self.spare = None
        self.room = torch.empty(256, dtype=torch.uint8, device=DEV)

    def _new_cache(self):
        held = [self.pool.take(self.stride) for _ in range(self.requests)]
        cache = B.lora_cache(self.pool.pages, torch.tensor(held, dtype=torch.int32, device=DEV), torch.zeros(self.requests, dtype=torch.int32, device=DEV),
                             self.page, self.kv_heads, self.head_dim, self.limit, self.pool.weight)
        return cache

    def _set_lengths(self, lengths):
        self.lengths = list(lengths)
        self.cache.length.copy_(torch.tensor(self.lengths, dtype=torch.int32))

    def _parts(self, qkv):
        """Addresses of q, k and v in rows of the projection's output, and the rows' length"""
        at, e, D = qkv.data_ptr(), qkv.element_size(), self.head_dim
        return at, at + self.heads * D * e, at + (self.heads + self.kv_heads) * D * e, qkv.shape[1]

    def _attend(self, q, ldq, tokens, most, indptr, decay):
        need = B.lora_cache_workspace(self.cache, self.heads, tokens, most, decay >= 0)
        if need > self.room.numel():
            self.room = torch.empty(need, dtype=torch.uint8, device=DEV)
        o = torch.empty((tokens, self.heads * self.head_dim), dtype=torch.bfloat16, device=DEV)
        B.lora_cache_attention(self.cache, B.LORA_BF16, self.heads, tokens, most, indptr, q, ldq, o, o.shape[1], self.head_dim ** -0.5, decay, self.room,
                               self.room.numel())
        return o

    def prompts(self, x, lengths, adapters):
        """x [tokens, hidden], the requests' prompts one behind the other, none longer than the caches' limit"""
        if max(lengths) > self.limit:
            raise ValueError("a prompt is longer than the cache's limit")
        if self.cache is None:
            self.cache, self.spare = self._new_cache(), self._new_cache()
        qkv = self.qkv(x, lengths, adapters)
        q, k, v, ld = self._parts(qkv)
        offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        indptr = torch.from_numpy(offsets).to(DEV)
        plan = B.lora_attention_plan(offsets, None, self.heads, self.kv_heads, self.head_dim, B.LORA_BF16)
        o = torch.empty((x.shape[0], self.heads * self.head_dim), dtype=torch.bfloat16, device=DEV)
        B.lora_attention(plan, q, ld, k, ld, v, ld, o, o.shape[1], self.head_dim ** -0.5)
        self._set_lengths(lengths)
        B.lora_cache_append(self.cache, B.LORA_BF16, x.shape[0], max(lengths), indptr, k, ld, v, ld)
        # the last tokens of every prompt once more, over the cache: their weights are what eviction goes by
        last = np.concatenate([np.arange(b - min(n, self.window), b) for n, b in zip(lengths, offsets[1:])])
        few = [min(n, self.window) for n in lengths]
        some = qkv[torch.from_numpy(last).to(DEV), :self.heads * self.head_dim].contiguous()
        self._attend(some, some.shape[1], len(last), max(few), torch.from_numpy(np.concatenate([[0], np.cumsum(few)]).astype(np.int32)).to(DEV), 0.0)
        y = self.out(o, lengths, adapters)
        torch.cuda.current_stream().synchronize()              # (the plan is given back when the work that uses it is through)
        plan.destroy()
        return y

    def decode(self, x, adapters):
        """x [requests, hidden]: a token of every request"""
        if max(self.lengths) >= self.limit:
            self.evict()
        S = self.requests
        self.lengths = [n + 1 for n in self.lengths]
        self.cache.length.add_(1)
        qkv = self.qkv(x, [1] * S, adapters)
        q, k, v, ld = self._parts(qkv)
        B.lora_cache_append(self.cache, B.LORA_BF16, S, 1, None, k, ld, v, ld)
        o = self._attend(q, ld, S, 1, None, 1.0)
        return self.out(o, [1] * S, adapters)

    def evict(self):
        """Returns the slots that were kept, [requests, kv heads, budget]"""
        kept = torch.empty((self.requests, self.kv_heads, self.budget), dtype=torch.int32, device=DEV)
        B.lora_cache_evict(self.cache, self.spare, self.budget, self.recent, kept)
        self.cache, self.spare = self.spare, self.cache
        self.lengths = [min(n, self.budget) for n in self.lengths]
        return kept


class BeamLayer:
    """The same layer for requests of several beams each, and the selection behind it.  Sequence r * beams + b is beam b of request r; tables, lengths and
    free pages are the device's, so that a step needs no word from it."""

    def __init__(self, hidden, heads, kv_heads, head_dim, ranks, requests, beams, limit, vocab, page=64, chosen=0, end_token=-1, scale=2.0, seed=0):
        """limit: tokens that a beam may have; chosen: pages of its cache that a token attends to (0: all)"""
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.head_dim, self.page = hidden, heads, kv_heads, head_dim, page
        self.requests, self.beams, self.limit, self.vocab, self.chosen, self.end_token = requests, beams, limit, vocab, chosen, end_token
        self.qkv = Projection(hidden, (heads + 2 * kv_heads) * head_dim, ranks, scale, gen)
        self.out = Projection(heads * head_dim, hidden, ranks, scale, gen)
        self.embedding = (torch.randn((vocab, hidden), generator=gen, device=DEV) * hidden ** -0.5).bfloat16()
        rows, each = requests * beams, -(-limit // page)
        count = rows * each                                     # (as many as beams that share nothing have)

        def zeros(*size, dtype=torch.int32):
            return torch.zeros(size, dtype=dtype, device=DEV)
        self.table, self.length, self.users = zeros(rows, each), zeros(rows), zeros(count)
        self.pages = B.lora_pages(self.table, self.length, self.users, page, limit)
        store = zeros(count, kv_heads, B.lora_cache_page_bytes(page, head_dim), dtype=torch.uint8)
        self.cache = B.lora_cache(store, self.table, self.length, page, kv_heads, head_dim, limit)
        padded = 64 if head_dim <= 64 else 128 if head_dim <= 128 else 256
        self.bounds, self.steps = zeros(count, kv_heads, 2, padded, dtype=torch.int8), zeros(count, kv_heads, dtype=torch.float32)
        self.wanted, self.parent, self.token, self.granted, self.indptr = zeros(rows), zeros(rows), zeros(rows), zeros(rows), zeros(rows + 1)
        self.copies, self.score = zeros(rows, 2), zeros(rows, dtype=torch.float32)
        self.best = [zeros(rows, dtype=torch.float32), zeros(rows), zeros(rows)]
        self.list = zeros(rows, kv_heads, max(chosen, 1))
        need = [B.lora_pages_workspace(self.pages), B.lora_beam_workspace(requests, beams, vocab, beams), B.lora_beam_workspace(requests, 1, vocab, beams),
                B.lora_cache_workspace(self.cache, heads, rows, 1)]
        if chosen:
            need += [B.lora_cache_choose_workspace(self.cache, rows, 1), B.lora_cache_chosen_workspace(self.cache, heads, rows, 1, chosen)]
        self.room = zeros(max(256, *need), dtype=torch.uint8)

    _parts = AttentionLayer._parts

    def _grow(self, tokens):
        """Pages for `tokens` new tokens; what shared pages hold, into the pages that take their place"""
        B.lora_pages_resize(self.pages, self.wanted, tokens, self.granted, self.indptr, None, None, None, self.copies, self.room, self.room.numel())
        B.lora_cache_copy(self.cache, len(self.copies), self.copies)

    def _select(self, y, first=False):
        """Logits of the rows' last tokens, and the best continuations: what the beams become, their tokens and scores.  first: one row a request"""
        beams = 1 if first else self.beams
        logits = torch.empty((len(y), self.vocab), dtype=torch.bfloat16, device=DEV)
        B.lora_base_gemm(len(y), self.hidden, self.vocab, B.LORA_BF16, y, self.hidden, self.embedding, self.hidden, logits, self.vocab)
        B.lora_beam_select(B.LORA_BF16, self.requests, beams, self.vocab, logits, self.vocab, self.score, None if first else self.token, self.end_token,
                           self.beams, *self.best, self.room, self.room.numel())
        self.logits = logits
        score, parent, token = self.best
        # (beams behind a request's first step all come of its one sequence)
        self.parent.copy_(torch.where(parent >= 0, parent * self.beams, -1) if first else parent)
        self.token.copy_(token)
        self.score.copy_(score)
        B.lora_pages_fork(self.pages, self.parent, self.room, self.room.numel())

    def prompts(self, x, lengths, adapters):
        """x [tokens, hidden], the requests' prompts one behind the other.  Afterwards every request has its first beams: token, score, parent"""
        if len(lengths) != self.requests or len(adapters) != self.requests or min(lengths) < 1 or sum(lengths) != len(x):
            raise ValueError("a prompt of at least a token and an adapter for every request")
        if max(lengths) > self.limit:
            raise ValueError("a prompt is longer than the caches' limit")
        self.longest = max(lengths)
        self.adapters = [a for a in adapters for _ in range(self.beams)]
        qkv = self.qkv(x, lengths, adapters)
        q, k, v, ld = self._parts(qkv)
        offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        plan = B.lora_attention_plan(offsets, None, self.heads, self.kv_heads, self.head_dim, B.LORA_BF16)
        o = torch.empty((x.shape[0], self.heads * self.head_dim), dtype=torch.bfloat16, device=DEV)
        B.lora_attention(plan, q, ld, k, ld, v, ld, o, o.shape[1], self.head_dim ** -0.5)
        # (the requests that were here before are through: their pages come back in the same call)
        self.wanted.zero_()
        self._grow(0)
        self.wanted.view(self.requests, self.beams)[:, 0] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        self._grow(x.shape[0])
        B.lora_cache_append(self.cache, B.LORA_BF16, x.shape[0], max(lengths), self.indptr, k, ld, v, ld)
        if self.chosen:
            B.lora_cache_digest(self.cache, x.shape[0], max(lengths), self.indptr, self.bounds, self.steps)
        y = self.out(o, lengths, adapters)
        self.score.zero_()
        self._select(y[torch.from_numpy(offsets[1:].astype(np.int64) - 1).to(DEV)].contiguous(), first=True)
        torch.cuda.current_stream().synchronize()              # (the plan is given back when the work that uses it is through)
        plan.destroy()

    def step(self):
        """The beams' last tokens through the layer, and the best of what may follow.  Every beam gets a token, so there is none where one of them is at the limit"""
        if self.longest >= self.limit:                          # (rows go by the sequences' new tokens: one that is not granted would shift those behind it)
            raise ValueError("a beam is at the caches' limit")
        self.longest += 1
        S, H, D = self.requests * self.beams, self.heads, self.head_dim
        torch.add(self.length, 1, out=self.wanted)
        self._grow(S)
        qkv = self.qkv(self.embedding[self.token.clamp_min(0)], [1] * S, self.adapters)
        q, k, v, ld = self._parts(qkv)
        B.lora_cache_append(self.cache, B.LORA_BF16, S, 1, self.indptr, k, ld, v, ld)
        o = torch.zeros((S, H * D), dtype=torch.bfloat16, device=DEV)
        if self.chosen:
            B.lora_cache_digest(self.cache, S, 1, self.indptr, self.bounds, self.steps)
            B.lora_cache_choose(self.cache, B.LORA_BF16, H, S, 1, self.indptr, q, ld, self.bounds, self.steps, self.chosen, min(1, self.chosen - 1), 1, self.list, self.room,
                                self.room.numel())
            B.lora_cache_attention_chosen(self.cache, B.LORA_BF16, H, S, 1, self.indptr, q, ld, o, H * D, D ** -0.5, self.chosen, self.list, self.room, self.room.numel())
        else:
            B.lora_cache_attention(self.cache, B.LORA_BF16, H, S, 1, self.indptr, q, ld, o, H * D, D ** -0.5, -1.0, self.room, self.room.numel())
        self._select(self.out(o, [1] * S, self.adapters))


def main(argv=None):
    ap = argparse.ArgumentParser()
    for name, value in (("requests", 32), ("prompt", 512), ("steps", 64), ("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("limit", 600), ("budget", 512),
                        ("beams", 4), ("vocab", 32000), ("chosen", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    args = ap.parse_args(argv)
    if args.hidden % args.heads:
        ap.error("hidden has to be a multiple of heads")
    rng = np.random.default_rng(0)
    lengths = np.clip(rng.lognormal(np.log(args.prompt) - 0.125, 0.5, args.requests).round(), 1, args.limit).astype(int).tolist()
    ranks, adapters = [8, 16, 32, 64] * 4, rng.integers(0, 16, args.requests).tolist()
    layer = AttentionLayer(args.hidden, args.heads, args.kv_heads, args.hidden // args.heads, ranks, args.requests, args.limit, args.budget, args.budget // 8)
    x = torch.randn((sum(lengths), args.hidden), device=DEV).bfloat16()
    xs = torch.randn((args.requests, args.hidden), device=DEV).bfloat16()

    def timed(f, n):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(n):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t) / n * 1e6

    for _ in range(2):
        prompts = timed(lambda: layer.prompts(x, lengths, adapters), 1)
    held = sum(layer.lengths) * args.kv_heads * (layer.pool.pages.shape[2] // layer.page)
    layer.decode(xs, adapters)
    steps = timed(lambda: layer.decode(xs, adapters), args.steps)
    evict = timed(layer.evict, 1)
    print(f"prompts of {sum(lengths)} tokens: {prompts:.0f} us a layer; {held / 1e6:.1f} MB of keys and values held")
    print(f"decode step of {args.requests} requests: {steps:.1f} us a layer, evictions at {args.limit} tokens among them; eviction: {evict:.0f} us")
    if args.beams > 0:
        del layer
        search = BeamLayer(args.hidden, args.heads, args.kv_heads, args.hidden // args.heads, ranks, args.requests, args.beams, args.limit + args.steps + 2, args.vocab,
                           chosen=args.chosen)
        for _ in range(2):
            prompts = timed(lambda: search.prompts(x, lengths, adapters), 1)
        search.step()
        steps = timed(search.step, args.steps)
        print(f"beam search, {args.beams} beams, {args.vocab} tokens: prompts {prompts:.0f} us, a step {steps:.1f} us, layer, logits and selection; "
              f"{int((search.users > 0).sum())} pages in use, named {int(search.users.sum())} times")
    return 0


if __name__ == "__main__":
    sys.exit(main())
