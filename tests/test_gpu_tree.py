"""Trees of drafted tokens over the paged 8-bit cache against plain 64-bit references:
their rows, attention over the sequence and a node's ancestors, the accepted path."""
import random

import pytest
import torch

from paper_2308_13137_amd import oq
from tests import serve_ref as ref
from tests import tree_ref
from tests.serve_ref import f64
from tests.test_gpu_serve import Batch, i32, rand

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def chain(n):
    return list(range(-1, n - 1))


def star(n):
    return [-1] + [0] * (n - 1)


def some_tree(n, seed, roots=0.1):
    r = random.Random(seed)
    return [-1 if j == 0 or r.random() < roots else r.randrange(max(0, j - 6), j) for j in range(n)]


def some_path(parent, seed):
    """From a root some way down."""
    r = random.Random(seed)
    at = [j for j, p in enumerate(parent) if p < 0]
    path = []
    while at and (not path or r.random() < 0.8):
        path.append(r.choice(at))
        at = [j for j, p in enumerate(parent) if p == path[-1]]
    return path


class Trees(Batch):
    """A cache with plain copies of every sequence, stepped by trees."""

    def tree_rows(self, qkv, parents):
        """Q~, K~ and V of the nodes in the kernel's fp32 order."""
        H, Hkv, d = self.H, self.Hkv, self.d
        pos = torch.tensor([L + t for L, p in zip(self.len, parents) for t in tree_ref.depths(p)])
        x = qkv.float().view(len(qkv), H + 2 * Hkv, d)
        q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
        if self.rope is not None:
            cs, sn = (self.rope.cpu()[pos][:, None, :, j] for j in (0, 1))
            q, k = ref.turn32(q, cs, sn), ref.turn32(k, cs, sn)
        if self.s_a is not None:
            sa = self.s_a.cpu().view(Hkv, d)
            q, k = q / sa.repeat_interleave(H // Hkv, 0), k * sa
        return q.to(BF), k.to(BF), v.to(BF)

    def tree_step(self, parents, paths, pad=3, max_q=None, attend=True):
        H, Hkv, d = self.H, self.Hkv, self.d
        counts = [len(p) for p in parents]
        qkv = self.new(counts)
        T = len(qkv)
        full = torch.cat([qkv, torch.full((pad, qkv.shape[1]), float("nan")).to(self.dtype)]).cuda()
        length, qs, mq = i32(self.len), i32(self.starts(counts)), max_q or max(counts)
        parent = i32(sum(parents, []) + [77] * pad)
        want_q, want_k, want_v = self.tree_rows(qkv, parents)
        out = torch.full((T + pad, H * d), 7.0, dtype=BF, device="cuda")
        codes = [t.clone() for t in (self.cache.k_codes, self.cache.v_codes)]
        q = self.cache.append_tree(full[:, :H * d], full[:, H * d:(H + Hkv) * d], full[:, (H + Hkv) * d:], self.table,
                                   length, qs, mq, parent, rope=self.rope, s_a=self.s_a, slots=self.slots, out=out)
        assert q is out and torch.equal(q[:T].cpu().view(T, H, d), want_q) and (q[T:] == 7).all()
        # drafts close no page
        assert torch.equal(codes[0], self.cache.k_codes) and torch.equal(codes[1], self.cache.v_codes)
        at = self.starts(counts)
        if attend:
            o = torch.full((T + pad, H * d), 7.0, dtype=BF, device="cuda")
            _, lse = self.cache.attend_tree(q, self.table, length, qs, mq, parent, slots=self.slots, want_lse=True,
                                            out=o)
            assert (o[T:] == 7).all()
            for i, c in enumerate(counts):
                if not c:
                    continue
                rows = slice(at[i], at[i] + c)
                k, v = (torch.cat([x[i].values(), new[rows].float()]) for x, new in
                        ((self.k, want_k), (self.v, want_v)))
                r, tol, rl = tree_ref.attend64(want_q[rows], k, v, tree_ref.sees(parents[i], self.len[i]))
                err = (f64(o[rows]).view(c, H, d) - r).abs()
                assert (err <= tol).all(), (i, float((err / tol).max()))
                assert ((f64(lse)[:, rows] - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()
        width = max([1] + [len(p) for p in paths]) + 2
        self.cache.commit(i32([p + [99] * (width - len(p)) for p in paths]), i32([len(p) for p in paths]), self.table,
                          length, qs, mq, slots=self.slots)
        for i, p in enumerate(paths):
            keep = [at[i] + j for j in p]
            self.k[i].add(want_k[keep])
            self.v[i].add(want_v[keep])
        self.len = [a + len(p) for a, p in zip(self.len, paths)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2), (5, 1)])
def test_tree_steps(d, page, H, Hkv):
    """Prompts, then trees of every shape whose paths end pages, beside sequences without nodes."""
    b = Trees(3, H, Hkv, d, page, 700, seed=d + page + H)
    b.step([150, 1, 33], attend=False)
    for k, sizes in enumerate(([5, 1, 17], [0, page, 30], [page, 2, 9], [1, 1, 1], [31, page - 1, 0], [page, page, page])):
        parents = [some_tree(n, 10 * k + i) if i != k % 3 else chain(n) for i, n in enumerate(sizes)]
        paths = [some_path(p, k + i) if i != k % 3 else p and list(range(len(p))) for i, p in enumerate(parents)]
        b.tree_step(parents, paths)
    b.step([40, 1, 2])
    b.check_rows()


@pytest.mark.parametrize("dtype,rope,s_a", [(F32, True, True), (F32, True, False), (BF, False, False),
                                            (F32, False, True)])
def test_tree_inputs(dtype, rope, s_a):
    b = Trees(2, 4, 2, 128, 64, 400, seed=5, rope=rope, s_a=s_a, dtype=dtype)
    b.step([100, 7], attend=False)
    for k in range(3):
        parents = [some_tree(40, k), star(9)]
        b.tree_step(parents, [some_path(parents[0], k), [0, 5]])
    b.check_rows()


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (16, 2), (40, 8)])
def test_tree_rows(n, H, Hkv):
    """Row counts around the row tiles; trees that end in the second page of the window."""
    b = Trees(2, H, Hkv, 64, 128, 800, seed=n + H, s_a=False)
    b.step([295, 254 - n // 2], attend=False)
    p, q = some_tree(n, n, 0.02), some_tree(1 + n // 2, n + 1, 0.02)
    b.tree_step([p, q], [some_path(p, 1), some_path(q, 2)])
    b.check_rows()


@pytest.mark.parametrize("L", [0, 1, 31, 32, 33, 1000, 4095, 4096, 4097])
@pytest.mark.parametrize("tree", [[-1], chain(5), [-1, 0, 0, 1, 1, 2], star(32)])
def test_tree_behind_lengths(L, tree):
    b = Trees(1, 4, 2, 128, 32, 4300, seed=L, s_a=False)
    if L:
        b.step([L], attend=False)
    b.tree_step([tree], [some_path(tree, L)])
    b.tree_step([tree], [[]])
    b.tree_step([tree], [some_path(tree, L + 1)])
    b.check_rows()


def test_trees_over_ragged_lengths_split():
    b = Trees(5, 4, 1, 64, 64, 3000, seed=3)
    b.step([1, 2900, 40, 64, 700], attend=False)
    for n in (1, 3, 20):
        parents = [some_tree(max(1, n - i), 7 * n + i) for i in range(5)]
        b.tree_step(parents, [some_path(p, n) for p in parents], max_q=n + 2)
    b.check_rows()


def test_many_small_trees_beside_a_large_one():
    b = Trees(40, 8, 1, 64, 128, 300, seed=8, s_a=False)
    b.step([random.Random(i).randint(1, 130) for i in range(40)], attend=False)
    parents = [some_tree(120 if i == 17 else i % 4, i) for i in range(40)]
    b.tree_step(parents, [some_path(p, i) for i, p in enumerate(parents)])
    b.check_rows()


@pytest.mark.parametrize("H,Hkv,lengths,n_max", [(16, 16, (0, 90), 5), (32, 16, (1, 300), 32), (64, 8, (0, 600), 20),
                                                 (40, 8, (400, 410), 17)])
def test_short_sequences_share_workgroups(H, Hkv, lengths, n_max):
    """Whole tiles of many sequences in one share, and cuts near the ends of tiles."""
    r = random.Random(H)
    n = 70
    b = Trees(n, H, Hkv, 64, 32, 700, seed=H, s_a=False, rope=False)
    b.step([r.randint(*lengths) for _ in range(n)], attend=False)
    parents = [some_tree(r.randint(0, n_max), i) if i % 9 else [] for i in range(n)]
    parents[40] = some_tree(n_max, 3)
    b.tree_step(parents, [some_path(p, i) for i, p in enumerate(parents)])


@pytest.mark.parametrize("H,Hkv,n", [(4, 4, 1), (4, 4, 20), (16, 2, 6), (16, 2, 30)])
def test_a_chain_is_a_batch_of_new_tokens(H, Hkv, n):
    """Where no page fills up a chain's queries and rows are append's, bit for bit, and its outputs attend's
    but for the order of sums: each is off by half a rounding to bf16 and what the weights' 11 bits leave."""
    d, P, L = 64, 64, 133
    x = rand(1, L + n, (H + 2 * Hkv) * d, dtype=BF)
    rope = oq.rope_table(256, d)
    table, got = i32([[2, 0, 3]]), []
    for tree in (False, True):
        c = oq.KVCache(4, P, Hkv, d, 1)

        def split(r):
            return r[:, :H * d], r[:, H * d:(H + Hkv) * d], r[:, (H + Hkv) * d:]
        c.append(*split(x[:L]), table, i32([0]), i32([0, L]), L, rope=rope)
        args = (table, i32([L]), i32([0, n]), n)
        if tree:
            q = c.append_tree(*split(x[L:]), *args, i32(chain(n)), rope=rope)
            got.append((q, *c.attend_tree(q, *args, i32(chain(n)), want_lse=True), c.k_window, c.v_window))
        else:
            q = c.append(*split(x[L:]), *args, rope=rope)
            got.append((q, *c.attend(q, *args, want_lse=True), c.k_window, c.v_window))
    (q, o, lse, *w), (q2, o2, lse2, *w2) = got
    for a, b in zip((q, *w), (q2, *w2)):
        assert torch.equal(a, b)
    # a weight rounds to 11 bits on both sides, the result to 8, values are below 6 in size
    assert ((f64(o) - f64(o2)).abs() <= 2 * (ref.BF8 * f64(o).abs() + ref.F11 * 6) * 1.01).all()
    assert ((f64(lse) - f64(lse2)).abs() <= 1e-4).all()


@pytest.mark.parametrize("page,d", [(32, 64), (64, 128), (128, 128)])
def test_commit_is_an_append_of_the_path(page, d):
    """Codes, steps and window rows after several trees equal those of the kept tokens appended one by one."""
    Hkv, H = 2, 4
    x = rand(3, 900, (H + 2 * Hkv) * d, dtype=BF)
    rope = oq.rope_table(1024, d)
    table = torch.randperm(1024 // page, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(1, -1).cuda()

    def split(r):
        return r[:, :H * d], r[:, H * d:(H + Hkv) * d], r[:, (H + Hkv) * d:]
    a, b = (oq.KVCache(1024 // page, page, Hkv, d, 1) for _ in range(2))
    at = L = page // 2 + 1
    kept = []
    for c in (a, b):
        c.append(*split(x[:L]), table, i32([0]), i32([0, L]), L, rope=rope)
    for k in range(14):
        n = [page, 3, 1, page - 1, 20][k % 5]
        tree = chain(n) if k % 4 == 1 else some_tree(n, k, 0.05)
        path = list(range(n)) if k % 4 == 1 else some_path(tree, k)
        rows = x[at:at + n]
        at = at + n if at + 2 * page < 900 else page
        a.append_tree(*split(rows), table, i32([L]), i32([0, n]), n, i32(tree), rope=rope)
        a.commit(i32([path]), i32([len(path)]), table, i32([L]), i32([0, n]), n)
        for j in path:
            b.append(*split(rows[j:j + 1]), table, i32([L]), i32([0, 1]), 1, rope=rope)
            L += 1
        for s, t in ((a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(s, t), k
        r, half = L % page, (L // page) % 2
        assert torch.equal(a.k_window[0, half, :, :r * d], b.k_window[0, half, :, :r * d])
        va, vb = (torch.stack([c.v_window[0, half].view(Hkv, page // 32, d // 16, 4, 16, 2, 4)]) for c in (a, b))
        t = torch.arange(page, device="cuda").view(page // 32, 2, 4, 4).permute(0, 2, 1, 3)       # chunk, g, e / 4, e % 4
        keep = (t < r)[None, None, :, None, :, None].expand(1, Hkv, page // 32, d // 16, 4, 16, 2, 4)
        assert torch.equal(va[keep], vb[keep])


def test_nodes_do_not_touch_others():
    """A node's key and value of any size, NaN and infinities among them, reach its descendants only."""
    H, Hkv, d, P = 8, 1, 64, 32
    for n, L in ((6, 40), (30, 61)):
        tree = some_tree(n, 5, 0.0)
        x = rand(n, L + n, (H + 2) * d, dtype=BF)
        table = i32([[0, 1, 2, 3]])
        outs = []
        for bad in (None, float("nan"), float("inf"), -float("inf"), 3e38):
            for col in (H * d + 3, (H + 1) * d + 9):
                y = x.clone()
                node = n // 2
                if bad is not None:
                    y[L + node, col] = bad
                c = oq.KVCache(4, P, Hkv, d, 1)
                c.append(y[:L, :H * d], y[:L, H * d:(H + 1) * d], y[:L, (H + 1) * d:], table, i32([0]), i32([0, L]), L)
                args = (table, i32([L]), i32([0, n]), n, i32(tree))
                r = y[L:]
                q = c.append_tree(r[:, :H * d], r[:, H * d:(H + 1) * d], r[:, (H + 1) * d:], *args)
                o = c.attend_tree(q, *args)
                outs.append(o)
                see = tree_ref.sees(tree, 0)[:, node].cuda()
                if bad is not None:
                    assert torch.equal(o[~see], outs[0][~see]), (n, bad, col)
                    if bad != 3e38:
                        assert torch.isnan(o[see].float()).all(), (n, bad, col)
                else:
                    assert torch.isfinite(o.float()).all()


@pytest.mark.parametrize("n,H", [(3, 4), (20, 2), (32, 8)])
def test_a_page_that_stands_for_nan(n, H):
    """Every node of a sequence sees its full pages: one that is NaN makes them all NaN."""
    d, P, L = 64, 32, 100
    x = rand(2, 2 * (L + n), (H + 2) * d, dtype=BF)
    x[10, H * d] = float("nan")
    c = oq.KVCache(8, P, 1, d, 2)
    table, parent = i32([[0, 1, 2, 3, 7], [4, 5, 6, 7, 7]]), i32(some_tree(n, 1) * 2)

    def split(r):
        return r[:, :H * d], r[:, H * d:(H + 1) * d], r[:, (H + 1) * d:]
    c.append(*split(x[:2 * L]), table, i32([0, 0]), i32([0, L, 2 * L]), L)
    args = (table, i32([L, L]), i32([0, n, 2 * n]), n, parent)
    q = c.append_tree(*split(x[2 * L:]), *args)
    o = c.attend_tree(q, *args)
    assert torch.isnan(o[:n].float()).all() and torch.isfinite(o[n:].float()).all()


def test_trees_that_do_not_fit():
    """Bad parents, slots, lengths and row ranges: NaN rows, nothing written or kept, others untouched."""
    d, P, n = 64, 32, 12
    cache = oq.KVCache(20, P, 1, d, 8)
    cache.k_window.fill_(3.0)
    cache.v_window.fill_(4.0)
    table = torch.arange(20, dtype=torch.int32, device="cuda").view(10, 2)
    x = rand(1, 10 * n, 3 * d, dtype=BF)
    slots = i32([0, 1, 2, 3, -1, 8, 4, 5, 6, 7])
    length = i32([20, 0, 0, 0, 0, 0, 60, -1, 20, 20])        # the seventh passes its two pages, the eighth is none
    trees = [chain(n) for _ in range(10)]
    trees[1][5], trees[2][0], trees[3][11] = 5, 0, -2        # itself, itself, no node
    qs = i32([n * i for i in range(10)] + [10 * n - 1])      # (the last one has a row less)
    parent = i32(sum(trees, []))
    before = [t.clone() for t in (cache.k_codes, cache.k_scale, cache.k_window, cache.v_window)]
    args = (table, length, qs, n)
    out = torch.full((10 * n, d), 7.0, dtype=BF, device="cuda")
    o = out.clone()
    cache.append_tree(x[:, :d], x[:, d:2 * d], x[:, 2 * d:], *args, parent, slots=slots, out=out)
    cache.attend_tree(torch.nan_to_num(out), *args, parent, slots=slots, out=o)
    for t in (out, o):
        t = t.view(10, n, d).float()
        assert torch.isfinite(t[0]).all() and torch.isnan(t[1:8]).all() and torch.isfinite(t[8]).all()
        assert torch.isfinite(t[9, :-1]).all() and (t[9, -1] == 7).all()
    for w, k in ((cache.k_window, 2), (cache.v_window, 3)):
        assert torch.equal(w[1:6], before[k][1:6])
    # paths that are none
    mid = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.k_window, cache.v_window)]
    path = torch.arange(n, dtype=torch.int32).repeat(10, 1)
    path[0, 3], path[8, 0], path[9, n - 1] = 2, -1, 11
    count = [n] * 10
    count[1] = count[2] = count[3] = -1
    cache.commit(path.cuda(), i32(count), *args, slots=slots)
    cache.commit(path[:, :n - 1].contiguous().cuda(), i32(count), *args, slots=slots)       # counts that pass the path
    cache.commit(path.cuda(), i32([n + 1] * 10), *args, slots=slots)                        # and the tree
    cache.commit(path.cuda(), i32([0] * 10), *args, slots=slots)
    for a, b in zip(mid, (cache.k_codes, cache.v_codes, cache.k_scale, cache.k_window, cache.v_window)):
        assert torch.equal(a, b)
    # a page outside the pool is not written when it fills up
    table[0, 0] = 20
    cache.commit(torch.arange(n, dtype=torch.int32).repeat(10, 1).cuda(), i32([n] + [0] * 9), *args, slots=slots)
    assert torch.equal(mid[0], cache.k_codes) and torch.equal(mid[2], cache.k_scale)


def test_tree_in_place_and_empty():
    H, d, P = 4, 64, 32
    c = oq.KVCache(4, P, 1, d, 1)
    x = rand(1, 6, (H + 2) * d, dtype=BF)
    args = (i32([[0, 1]]), i32([0]), i32([0, 6]), 6, i32([-1, 0, 0, 1, 1, 2]))
    q0 = x[:, :H * d].contiguous()
    k, v = x[:, H * d:(H + 1) * d], x[:, (H + 1) * d:]
    rope = oq.rope_table(64, d)
    want = c.append_tree(q0, k, v, *args, rope=rope)
    o = c.attend_tree(want, *args)
    q = q0.clone()
    assert c.append_tree(q, k, v, *args, rope=rope, out=q) is q and torch.equal(q, want)
    assert torch.equal(c.attend_tree(q, *args, out=q), o)
    none = (i32([[0, 1]]), i32([0]), i32([0, 0]), 0, i32([]))
    assert c.append_tree(q0[:0], k[:0], v[:0], *none).shape == (0, H * d)
    assert c.attend_tree(q0[:0], *none).shape == (0, H * d)
    # rotations past the table
    q = c.append_tree(q0, k, v, *args, rope=oq.rope_table(2, d))
    deep = torch.tensor(tree_ref.depths([-1, 0, 0, 1, 1, 2])) >= 2
    assert torch.isnan(q[deep.cuda()].float()).all() and torch.equal(q[~deep.cuda()], want[~deep.cuda()])


def test_windows_past_32_bits():
    """The last of 8,200 windows, whose elements lie behind 2^31."""
    Hkv, d, P = 8, 128, 128
    n_slots = 2 ** 31 // (2 * Hkv * P * d) + 8
    assert n_slots * 2 * Hkv * P * d > 2 ** 31
    blk = P * d
    shape = (n_slots, 2, Hkv, blk)
    kw, vw = (torch.empty(shape, dtype=BF, device="cuda") for _ in range(2))
    c = oq.KVCache.of(*(torch.zeros(4, Hkv, blk, dtype=torch.int8, device="cuda") for _ in range(2)),
                      *(torch.zeros(4, Hkv, device="cuda") for _ in range(2)), kw, vw, P, d)
    s = oq.KVCache(4, P, Hkv, d, 1)
    x = rand(1, 150, (16 + 2 * Hkv) * d, dtype=BF)

    def split(r):
        return r[:, :16 * d], r[:, 16 * d:(16 + Hkv) * d], r[:, (16 + Hkv) * d:]
    table, tree = i32([[0, 1, 2]]), some_tree(30, 4)
    got = []
    for cache, slots in ((c, i32([n_slots - 1])), (s, None)):
        cache.append(*split(x[:120]), table, i32([0]), i32([0, 120]), 120, slots=slots)
        args = (table, i32([120]), i32([0, 30]), 30)
        q = cache.append_tree(*split(x[120:]), *args, i32(tree), slots=slots)
        o = cache.attend_tree(q, *args, i32(tree), slots=slots)
        path = [0, 4, 7, 9, 11, 12, 20, 21, 29]
        cache.commit(i32([path]), i32([9]), *args, slots=slots)
        got.append((q, o, cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, cache.k_window[-1, 1, :, :d]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
