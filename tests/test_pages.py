"""Pages given out, taken back, shared and copied on the device, against the definitions of include/lora_abi.h one sequence after the other, and
what the calls refuse.  All results are whole numbers, or copied bits, and have to be equal."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B

DEV = "cuda:0"
gpu = pytest.mark.gpu


def count(tokens, page):
    return -(-tokens // page)


class Model:
    """The definitions, step by step"""

    def __init__(self, table, length, users, page, max_length):
        self.table, self.length, self.users, self.page, self.max = table.copy(), length.copy(), users.copy(), page, max_length

    def known(self, p):
        return 0 <= p < len(self.users)

    def resize(self, wanted):
        P, S = self.page, len(self.length)
        L = np.clip(self.length, 0, self.max)
        fits = [0 <= w <= self.max for w in wanted]
        W = [int(w) if f else int(n) for w, f, n in zip(wanted, fits, L)]
        for s in range(S):
            for e in range(count(W[s], P), count(int(L[s]), P)):
                if self.known(self.table[s, e]):
                    self.users[self.table[s, e]] -= 1
                self.table[s, e] = -1
        sharers = {}
        for s in range(S):
            if W[s] > L[s] and L[s] % P:
                p = self.table[s, L[s] // P]
                if self.known(p) and self.users[p] > 1:
                    sharers.setdefault(int(p), []).append(s)
        copying = set()
        for p, who in sharers.items():
            keeper = max(who, key=lambda s: (L[s] % P, s)) if len(who) == self.users[p] else None
            copying |= set(who) - {keeper}
        free = [p for p in range(len(self.users)) if self.users[p] == 0]
        granted, copies, indptr, new, short = [], [], [0], [], False
        left = {p: len(set(who) & copying) for p, who in sharers.items()}
        for s in range(S):
            grows = W[s] > L[s]
            need = count(W[s], P) - count(int(L[s]), P) + (s in copying) if grows else 0
            served = need == 0 or (not short and need <= len(free))
            short |= not served
            copies.append((-1, -1))
            granted.append(int(served and fits[s]))
            if served and need:
                mine, free = free[:need], free[need:]
                if s in copying:
                    e = L[s] // P
                    copies[-1] = (int(self.table[s, e]), mine[0])
                    self.users[self.table[s, e]] -= 1
                    self.table[s, e], mine = mine[0], mine[1:]
                    self.users[self.table[s, e]] = 1
                for e, p in zip(range(count(int(L[s]), P), count(W[s], P)), mine):
                    self.table[s, e] = p
                    self.users[p] = 1
            if served and fits[s]:
                self.length[s] = W[s]
            if served and grows:
                for i in range(int(L[s]), W[s]):
                    p = self.table[s, i // P]
                    new.append((s, i, int(p) * P + i % P if self.known(p) else -1))
            indptr.append(len(new))
        return granted, indptr, new, copies

    def fork(self, parent):
        S, stride = self.table.shape
        L = np.clip(self.length, 0, self.max)
        old, table, length = self.table, self.table.copy(), self.length.copy()
        for s in range(S):
            p = parent[s]
            if p == s:
                continue
            there = 0 <= p < S
            n = count(int(L[p]), self.page) if there else 0
            for e in range(stride):
                table[s, e] = old[p, e] if e < n else -1
            length[s] = L[p] if there else 0
            for e in range(count(int(L[s]), self.page)):
                if self.known(old[s, e]):
                    self.users[old[s, e]] -= 1
            for e in range(n):
                if self.known(table[s, e]):
                    self.users[table[s, e]] += 1
        self.table, self.length = table, length


class State:
    """A model, and the same on the device"""

    def __init__(self, S, stride, num_pages, page, max_length=None, rng=None, held=0):
        table, length, users = np.full((S, stride), -1, np.int32), np.zeros(S, np.int32), np.zeros(num_pages, np.int32)
        if rng is not None:
            table[:] = rng.integers(-5, 2 ** 31 - 1, table.shape)            # (what is behind a sequence's pages is anything)
            users[rng.permutation(num_pages)[:held]] = 1
        self.max = stride * page if max_length is None else max_length
        self.m = Model(table, length, users, page, self.max)
        self.table, self.length, self.users = (torch.from_numpy(x.copy()).to(DEV) for x in (table, length, users))
        self.pages = B.lora_pages(self.table, self.length, self.users, page, self.max)
        self.room = torch.full((max(256, B.lora_pages_workspace(self.pages)),), 0xff, dtype=torch.uint8, device=DEV)
        self.S = S

    def resize(self, wanted, rows=None, check=True):
        granted, indptr, new, copies = self.m.resize(wanted)
        rows = len(new) if rows is None else rows
        guard = 3
        d = {k: torch.full((n + guard,), -9, dtype=t, device=DEV) for k, n, t in (("granted", self.S, torch.int32), ("indptr", self.S + 1, torch.int32),
             ("seq", rows, torch.int32), ("position", rows, torch.int32), ("slot", rows, torch.int64), ("copies", 2 * self.S, torch.int32))}
        B.lora_pages_resize(self.pages, torch.from_numpy(np.asarray(wanted, np.int32)).to(DEV), rows, d["granted"], d["indptr"], d["seq"], d["position"], d["slot"],
                            d["copies"], self.room, self.room.numel())
        torch.cuda.synchronize()
        got = {k: x.cpu().numpy() for k, x in d.items()}
        fill = lambda x, n: list(x[:n]) + [-9] * (n - len(x[:n]))  # noqa: E731
        expect = {"granted": granted, "indptr": indptr, "copies": [p for c in copies for p in c], "seq": fill([t[0] for t in new], rows),
                  "position": fill([t[1] for t in new], rows), "slot": fill([t[2] for t in new], rows)}
        for k, x in expect.items():
            assert got[k].tolist() == x + [-9] * guard, k
        self.check()
        return copies

    def fork(self, parent):
        self.m.fork(parent)
        B.lora_pages_fork(self.pages, torch.from_numpy(np.asarray(parent, np.int32)).to(DEV), self.room, self.room.numel())
        torch.cuda.synchronize()
        self.check()

    def check(self):
        assert np.array_equal(self.length.cpu().numpy(), self.m.length)
        table = self.table.cpu().numpy()
        bad = np.argwhere(table != self.m.table)
        assert len(bad) == 0, (bad[:4], [(table[tuple(b)], self.m.table[tuple(b)]) for b in bad[:4]])
        assert np.array_equal(self.users.cpu().numpy(), self.m.users)


# sequences, entries each, pages, tokens a page: one workgroup for all; three launches; threads of several sequences
SHAPES = [(1, 1, 1, 32), (1, 40, 30, 32), (5, 3, 9, 64), (37, 20, 400, 32), (1000, 4, 2500, 64), (300, 130, 20000, 32), (1024, 8, 6000, 96), (2, 3000, 5000, 32), (1025, 3, 2000, 32),
          (4500, 5, 12000, 64), (16384, 2, 20001, 32)]


@gpu
@pytest.mark.parametrize("S,stride,num_pages,page", SHAPES)
def test_sequences_come_grow_share_and_go(S, stride, num_pages, page):
    rng = np.random.default_rng(S + stride)
    st = State(S, stride, num_pages, page, rng=rng, held=num_pages // 7)
    top = st.max
    mean = max(1, min(top, num_pages * page // (S + 1)))
    for step in range(9):
        now = np.clip(st.m.length, 0, top)
        kind = rng.integers(0, 6, S)
        wanted = np.select([kind == 0, kind == 1, kind == 2, kind == 3], [now + 1, 0, rng.integers(0, top + 1, S), now + rng.integers(0, 2 * page, S)], now)
        if step % 3 == 1:
            wanted = np.where(rng.random(S) < 0.05, rng.choice([-1, top + 1, -2 ** 31, 2 ** 31 - 1], S), wanted)
        if step == 0:
            wanted = np.minimum(top, rng.integers(0, 2 * mean, S))
        st.resize(np.clip(wanted, -2 ** 31, 2 ** 31 - 1), rows=None if step % 4 else 100)
        if step % 2:
            near = np.arange(S) // 4 * 4 + rng.integers(0, 4, S)
            st.fork(np.where(rng.random(S) < 0.03, rng.choice([-1, S, -2 ** 31, 2 ** 31 - 1], S), np.where(near < S, near, 0)))
            st.resize(np.minimum(st.m.length + 1, top))


@gpu
@pytest.mark.parametrize("S", [8, 2000])
@pytest.mark.parametrize("room", [0, 1, 3])
def test_pages_shared_by_all_that_grow(S, room):
    """Eight beams of one prompt that ends inside a page: one keeps the page, others get copies as long as there are pages"""
    page = 64
    st = State(S, 4, 3 + room, page)
    st.resize([130] + [0] * (S - 1))
    st.fork([0] * 8 + list(range(8, S)))
    copies = st.resize([131] * 8 + [0] * (S - 8))
    assert [c[0] >= 0 for c in copies[:8]].count(True) == min(7, room) and copies[7] == (-1, -1)
    st.resize([0] * S)
    assert (st.users == 0).all()


@gpu
def test_the_one_with_the_most_tokens_keeps_the_page():
    st = State(4, 3, 6, 32)
    st.resize([40, 0, 0, 0])
    st.fork([0, 0, 0, 3])
    st.resize([35, 40, 33, 0])                              # (two are cut within the page)
    copies = st.resize([64, 41, 34, 0])
    assert copies[1] == (-1, -1) and copies[0][0] == copies[2][0] >= 0
    st.fork([1, 1, 1, 1])
    copies = st.resize([41, 42, 0, 41])                     # some stay: whoever grows gets a copy
    assert copies[1][0] >= 0


@gpu
@pytest.mark.parametrize("S", [3, 1500])
def test_entries_that_are_not_there(S):
    st = State(S, 4, 60, 32)
    wanted = [100, 70, 33] + [0] * (S - 3)
    st.resize(wanted)
    for s, e, p in ((0, 1, -1), (0, 3, 60), (1, 0, 2 ** 31 - 1), (2, 1, -7)):
        st.table[s, e] = st.m.table[s, e] = p
    st.resize([101, 128, 34] + [0] * (S - 3))
    st.fork([1, 0, 2] + list(range(3, S)))
    st.resize([0] * S)


@gpu
def test_more_new_pages_than_are_kept_near():
    """One workgroup, and a list of free pages that is longer than it holds itself"""
    st = State(4, 6000, 13000, 32, rng=np.random.default_rng(3), held=900)
    st.resize([5000 * 32, 33, 4000 * 32 + 1, 6000 * 32], rows=16000)
    st.resize([0, 34, 4000 * 32 + 40, 5000 * 32 + 7], rows=16000)


@gpu
@pytest.mark.parametrize("S", [5, 1500])
def test_a_table_without_entries_and_a_pool_without_pages(S):
    st = State(S, 0, 3, 32)
    st.resize(np.arange(S) % 2)                             # (nothing may be longer than 0)
    st.fork(np.arange(S)[::-1])
    st = State(S, 2, 0, 32)
    st.resize(np.arange(S) % 40)
    st.fork(np.arange(S)[::-1])


@gpu
def test_what_is_not_wanted_is_left_out():
    st = State(3, 4, 20, 32)
    wanted, copies = torch.tensor([40, 0, 70], dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    B.lora_pages_resize(st.pages, wanted, 1000, None, None, None, None, None, copies, st.room, st.room.numel())
    st.m.resize([40, 0, 70])
    st.check()
    slot = torch.full((120,), -5, dtype=torch.int64, device=DEV)
    B.lora_pages_resize(st.pages, wanted + 5, 16, None, None, None, None, slot, copies, st.room, st.room.numel())
    _, _, new, _ = st.m.resize([45, 5, 75])
    st.check()
    assert slot.tolist() == [t[2] for t in new] + [-5] * 105


@gpu
@pytest.mark.parametrize("S,stride", [(6, 4), (1300, 3)])
def test_a_captured_step_of_beams(S, stride):
    """fork and resize as a graph, replayed with other parents and lengths, eager work in between; each replay against the model"""
    page, rng = 32, np.random.default_rng(5)
    st = State(S, stride, 3 * S + 9, page)
    st.resize(rng.integers(1, 2 * page, S))
    parent, wanted = (torch.zeros(S, dtype=torch.int32, device=DEV) for _ in range(2))
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (S, S + 1, S, S, 2 * S)]
    slot = torch.zeros(S, dtype=torch.int64, device=DEV)
    parent.copy_(torch.arange(S))
    wanted.copy_(st.length)

    def step():
        B.lora_pages_fork(st.pages, parent, st.room, st.room.numel())
        B.lora_pages_resize(st.pages, wanted, S, out[0], out[1], out[2], out[3], slot, out[4], st.room, st.room.numel())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        p = np.arange(S) // 3 * 3 + rng.integers(0, 3, S)
        p = np.where(p < S, p, 0)
        st.m.fork(p)
        w = np.minimum(st.m.length + 1, st.max)
        granted, indptr, new, copies = st.m.resize(w)
        parent.copy_(torch.from_numpy(p.astype(np.int32)))
        wanted.copy_(torch.from_numpy(w.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        st.check()
        assert out[0].tolist() == granted and out[1].tolist() == indptr and out[4].view(-1, 2).tolist() == [list(c) for c in copies]
        assert slot[:len(new)].tolist() == [t[2] for t in new]
        torch.ones(1000, device=DEV).sum()


@gpu
@pytest.mark.parametrize("D,page,heads", [(64, 32, 1), (128, 64, 8), (80, 96, 3), (256, 32, 2)])
@pytest.mark.parametrize("weight", [True, False])
def test_pages_are_copied(D, page, heads, weight):
    rng, n = np.random.default_rng(D), 40
    raw = torch.from_numpy(rng.integers(0, 256, (n, heads, B.lora_cache_page_bytes(page, D)), dtype=np.uint8)).to(DEV)
    w = torch.from_numpy(rng.standard_normal((n, heads, page)).astype(np.float32)).to(DEV) if weight else None
    cache = B.lora_cache(raw.clone(), torch.zeros((2, 4), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), page, heads, D, 64,
                         None if w is None else w.clone())
    copies = [(3, 20), (-1, -1), (5, 21), (3, 22), (7, -1), (-1, 23), (8, n), (n, 24), (9, 9), (10, 39), (2 ** 31 - 1, 25)]
    B.lora_cache_copy(cache, len(copies), torch.tensor(copies, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for a, b in ((3, 20), (5, 21), (3, 22), (10, 39)):
        raw[b] = raw[a]
        if weight:
            w[b] = w[a]
    assert torch.equal(cache.pages, raw) and (not weight or torch.equal(cache.weight, w))


@gpu
def test_a_cache_beyond_4_gb_is_copied():
    page, D, heads = 64, 128, 8
    size = B.lora_cache_page_bytes(page, D)
    n = (1 << 32) // (heads * size) + 40
    pages = torch.zeros((n, heads, size), dtype=torch.uint8, device=DEV)
    pages[n - 1] = torch.arange(size, device=DEV).to(torch.uint8)
    pages[3] = 7
    cache = B.lora_cache(pages, torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV), page, heads, D, 64)
    B.lora_cache_copy(cache, 2, torch.tensor([[n - 1, 5], [3, n - 2]], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(pages[5], pages[n - 1]) and (pages[n - 2] == 7).all() and (pages[4] == 0).all() and (pages[n - 3] == 0).all()


# ---- refusals (no GPU) ---------------------------------------------------------------------------------------------------
OK, BAD, UNSUPPORTED, WORKSPACE = B.LORA_OK, B.LORA_ERR_INVALID_ARG, B.LORA_ERR_UNSUPPORTED, B.LORA_ERR_WORKSPACE
FINE = dict(page_table=1 << 20, length=2 << 20, users=3 << 20, num_pages=1000, num_seqs=16, table_stride=10, max_length=600, page_tokens=64)


def desc(**f):
    return B.PagesDesc(*[{**FINE, **f}[n] for n, _ in B.PagesDesc._fields_])


def status(call, *args):
    try:
        call(*args)
    except B.LoraError as e:
        return e.status
    return OK


WRONG = [(dict(num_seqs=-1), BAD), (dict(num_pages=-1), BAD), (dict(table_stride=-1), BAD), (dict(max_length=-1), BAD), (dict(max_length=641), BAD), (dict(page_tokens=33), BAD),
         (dict(page_tokens=0), BAD), (dict(page_tokens=2048), BAD), (dict(length=0), BAD), (dict(page_table=0), BAD), (dict(users=0), BAD), (dict(length=(2 << 20) + 2), BAD),
         (dict(users=(3 << 20) + 1), BAD), (dict(page_table=(1 << 20) + 3), BAD), (dict(num_seqs=(1 << 14) + 1), UNSUPPORTED), (dict(num_pages=1 << 31), UNSUPPORTED),
         (dict(num_pages=(1 << 25) - 10), UNSUPPORTED), (dict(table_stride=1 << 25, max_length=(1 << 30) + 1), UNSUPPORTED),
         (dict(num_seqs=1 << 14, table_stride=1 << 18), UNSUPPORTED)]


@pytest.mark.parametrize("fields,expected", WRONG)
def test_descriptors_are_refused(fields, expected):
    p = B.Pages(desc(**fields))
    assert status(B.lora_pages_workspace, p) == expected
    assert status(B.lora_pages_resize, p, 4 << 20, 100, None, None, None, None, None, 5 << 20, 6 << 20, 1 << 40, 1) == expected
    assert status(B.lora_pages_fork, p, 4 << 20, 6 << 20, 1 << 40, 1) == expected


def test_calls_are_refused():
    p = B.Pages(desc())
    need = B.lora_pages_workspace(p)
    assert need == -(-(16 * 16 + 256 + 1000 * 4) // 256) * 256                     # (what a sequence gets, parts of the pool, free pages)
    fine = dict(d_wanted=4 << 20, num_tokens=100, d_granted=7 << 20, d_indptr=8 << 20, d_token_seq=9 << 20, d_token_position=10 << 20, d_token_slot=11 << 20,
                d_copies=5 << 20, workspace=6 << 20, workspace_bytes=need)
    resize = lambda **f: status(lambda: B.lora_pages_resize(p, **{**fine, **f}, stream=1))  # noqa: E731
    for f in (dict(num_tokens=-1), dict(d_wanted=None), dict(d_copies=None), dict(d_wanted=(4 << 20) + 2), dict(d_granted=(7 << 20) + 1), dict(d_indptr=(8 << 20) + 2),
              dict(d_token_seq=(9 << 20) + 2), dict(d_token_position=(10 << 20) + 1), dict(d_token_slot=(11 << 20) + 4), dict(d_copies=(5 << 20) + 2)):
        assert resize(**f) == BAD, f
    for f in (dict(workspace=None), dict(workspace=(6 << 20) + 128), dict(workspace_bytes=need - 1)):
        assert resize(**f) == WORKSPACE, f
        assert status(lambda: B.lora_pages_fork(p, 4 << 20, **{**dict(workspace=6 << 20, workspace_bytes=need), **f}, stream=1)) == WORKSPACE
    # outputs that lie on what is read, or on each other
    for f in (dict(d_granted=4 << 20), dict(d_granted=(4 << 20) + 60), dict(d_indptr=(1 << 20) + 636), dict(d_token_seq=(2 << 20) - 396), dict(d_token_slot=(3 << 20) + 3992),
              dict(d_copies=4 << 20), dict(d_copies=(6 << 20) + need - 4), dict(d_token_position=(9 << 20) + 396), dict(workspace=(2 << 20) - 256), dict(d_wanted=2 << 20),
              dict(d_wanted=(6 << 20) - 60)):
        assert resize(**f) == BAD, f
    assert status(lambda: B.lora_pages_fork(p, None, 6 << 20, need, 1)) == BAD
    for parent in ((4 << 20) + 1, 2 << 20, 3 << 20, (1 << 20) + 100, 6 << 20):
        assert status(lambda: B.lora_pages_fork(p, parent, 6 << 20, need, 1)) == BAD
    none = B.Pages(desc(num_seqs=0, page_table=0, length=0, users=0))
    assert B.lora_pages_workspace(none) == 0
    assert status(lambda: B.lora_pages_resize(none, None, 0, None, None, None, None, None, None, None, 0, 1)) == OK
    assert status(lambda: B.lora_pages_fork(none, None, None, 0, 1)) == OK


def test_copies_are_refused():
    c = B.Cache(B.CacheDesc(1 << 20, None, 2 << 20, 3 << 20, 100, 4, 10, 640, 64, 8, 128))
    for args, expected in (((-1, 4 << 20), BAD), ((5, None), BAD), ((5, (4 << 20) + 2), BAD), (((1 << 24) // 8, 4 << 20), UNSUPPORTED), ((0, None), OK)):
        assert status(lambda: B.lora_cache_copy(c, *args, 1)) == expected, args


def test_descriptors_are_made_of_fitting_tensors():
    table, length, users = (torch.zeros(n, dtype=torch.int32) for n in ((3, 5), 3, 7))
    p = B.lora_pages(table, length, users, 64, 100)
    assert (p.desc.num_pages, p.desc.num_seqs, p.desc.table_stride, p.desc.max_length, p.desc.page_tokens) == (7, 3, 5, 100, 64)
    for bad in (dict(page_table=table.long()), dict(page_table=table.t()), dict(page_table=table[0]), dict(length=length[:2]), dict(users=users.float()), dict(users=users[::2])):
        with pytest.raises(ValueError):
            B.lora_pages(**{**dict(page_table=table, length=length, users=users, page_tokens=64, max_length=100), **bad})


def test_the_descriptor_has_the_headers_layout(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "lora_abi.h"\nint main(void) { printf("%zu ", sizeof(lora_pages));' +
                   "".join(f'printf("%zu ", offsetof(lora_pages, {f}));' for f, _ in B.PagesDesc._fields_) + "return 0; }\n")
    subprocess.run(["gcc", "-I" + os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    assert out == [ctypes.sizeof(B.PagesDesc)] + [getattr(B.PagesDesc, f).offset for f, _ in B.PagesDesc._fields_]


P, I32, I64, F, Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
ABI = {"lora_pages_resize": [P, P, I32, P, P, P, P, P, P, P, Z, P], "lora_pages_fork": [P, P, P, Z, P], "lora_cache_copy": [P, I32, P, P],
       "lora_beam_select": [I32, I32, I32, I32, P, I64, P, P, I32, I32, P, P, P, P, Z, P], "lora_cache_digest": [P, I32, I32, P, P, P, P],
       "lora_cache_choose": [P, I32, I32, I32, I32, P, P, I64, P, P, I32, I32, I32, P, P, Z, P],
       "lora_cache_attention_chosen": [P, I32, I32, I32, I32, P, P, I64, P, I64, F, I32, P, P, Z, P]}


@pytest.mark.parametrize("calls", ["_calls", "calls_ctypes"])
@pytest.mark.parametrize("name", list(ABI))
def test_arguments_reach_the_abi(calls, name):
    """By position and by name, in place; what is missing or too much is refused"""
    import importlib
    import inspect
    import types
    module = importlib.import_module("paper_2411_00915_amd." + calls)
    seen, result = [], [0]
    keep = [ctypes.CFUNCTYPE(ctypes.c_int, *arguments)(lambda *a, n=n: (seen.append((n, list(a))), result[0])[1]) for n, arguments in ABI.items()]
    if calls == "calls_ctypes":
        module.bind(B._check, B._first_stream, *[B._address(keep[0])] * 8)
    module.bind_sequences(*(B._address(f) for f in keep))
    try:
        function = getattr(module, name)
        parameters = inspect.signature(function).parameters
        assert list(parameters) == list(inspect.signature(getattr(B, name)).parameters) and len(parameters) == len(ABI[name])
        values = {p: types.SimpleNamespace(handle=0x1000 + i) if p in ("pages", "cache") else 0.25 if p == "scale" else 64 + i for i, p in enumerate(parameters)}
        expected = [0x1000 + i if p in ("pages", "cache") else v for i, (p, v) in enumerate(values.items())]
        function(*values.values())
        function(**dict(reversed(values.items())))
        assert seen == [(name, expected)] * 2
        for wrong in (list(values.values())[:-2], [*values.values(), 0]):
            with pytest.raises(TypeError):
                function(*wrong)
        result[0] = B.LORA_ERR_WORKSPACE
        with pytest.raises(B.LoraError, match=f"{name}: workspace"):
            function(**values)
    finally:
        if calls == "_calls":
            module.bind_sequences(*(B._address(getattr(B._lib, n)) for n in ABI))


def test_the_definition_by_hand():
    m = Model(np.full((3, 4), -1, np.int32), np.zeros(3, np.int32), np.array([1, 0, 0, 0, 0, 0], np.int32), 32, 128)
    assert m.resize([33, 0, 200]) == ([1, 1, 0], [0, 33, 33, 33], [(0, i, 32 + i) for i in range(32)] + [(0, 32, 64)], [(-1, -1)] * 3)
    m.fork([0, 0, 2])
    assert m.table[1].tolist() == [1, 2, -1, -1] and m.users.tolist() == [1, 2, 2, 0, 0, 0]
    granted, _, new, copies = m.resize([34, 34, 0])
    assert copies == [(2, 3), (-1, -1), (-1, -1)] and new == [(0, 33, 97), (1, 33, 65)] and m.users.tolist() == [1, 2, 1, 1, 0, 0]
    assert m.resize([129, 128, 96])[0] == [0, 1, 0]
