"""Drafted tokens as a program uses them: whole steps of a decoder, captured into a graph, on
other streams, beside one that decodes token by token."""
import random

import pytest
import torch

from paper_2308_13137_amd import oq
from tests.test_gpu_serve import i32, rand
from tests.test_gpu_tree import chain, some_tree
from tests.test_gpu_tree import Trees

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


class Decoder:
    """One block's attention between an embedding and logits: n sequences of one cache."""

    def __init__(self, seed, n=3, H=8, Hkv=2, d=64, page=32, V=1003, pages=12):
        self.n, self.H, self.Hkv, self.d, self.V = n, H, Hkv, d, V
        self.embed = rand(seed, V, (H + 2 * Hkv) * d)
        self.head = rand(seed + 1, H * d, V, scale=2.0)
        self.cache = oq.KVCache(n * pages, page, Hkv, d, n)
        self.table = torch.randperm(n * pages, generator=torch.Generator().manual_seed(seed)).view(n, pages).int().cuda()
        self.rope = oq.rope_table(page * pages, d)
        self.length = torch.zeros(n, dtype=torch.int32, device="cuda")

    def split(self, token):
        x = self.embed[token.long()]
        a, b = self.H * self.d, (self.H + self.Hkv) * self.d
        return x[:, :a], x[:, a:b], x[:, b:]

    def logits(self, o):
        return o.float() @ self.head

    def prompt(self, tokens):
        m = len(tokens[0])
        t = torch.tensor(tokens, device="cuda").view(-1)
        args = (self.table, self.length, i32([m * i for i in range(self.n + 1)]), m)
        q = self.cache.append(*self.split(t), *args, rope=self.rope)
        o = self.cache.attend(q, *args)
        self.length += m
        return self.logits(o[m - 1::m]).argmax(1).int()

    def one(self, token):
        args = (self.table, self.length, i32(list(range(self.n + 1))), 1)
        q = self.cache.append(*self.split(token), *args, rope=self.rope)
        o = self.cache.attend(q, *args)
        self.length += 1
        return self.logits(o).argmax(1).int()

    def step(self, token, parent, q_start, max_q, temperature, u, u_next, Q=None):
        """A whole step over trees: (path, count, next token)."""
        args = (self.table, self.length, q_start, max_q)
        q = self.cache.append_tree(*self.split(token), *args, parent, rope=self.rope)
        o = self.cache.attend_tree(q, *args, parent)
        P = oq.token_probs(self.logits(o), temperature)
        path, count, nxt = oq.tree_verify(token, parent, q_start, max_q, P, u, u_next, Q=Q)
        self.cache.commit(path, count, *args)
        self.length += count
        return path, count, nxt


def rows_of(dec):
    """Every cached row of a decoder, as values."""
    n, L = dec.n, dec.length.tolist()
    start = [0]
    for x in L:
        start.append(start[-1] + x)
    return dec.cache.read(dec.table, i32([0] * n), dec.length, i32([0] * (n + 1)), i32(start), start[-1], max(L), dtype=F32)


class Step:
    """A step's inputs in fixed buffers, for graphs."""

    def __init__(self, dec, seed, nodes=9):
        self.dec, self.nodes = dec, nodes
        T = dec.n * nodes
        self.token, self.parent = (torch.zeros(T, dtype=torch.int32, device="cuda") for _ in range(2))
        self.q_start = i32([nodes * i for i in range(dec.n + 1)])
        self.u, self.u_next = torch.zeros(T, device="cuda"), torch.zeros(dec.n, device="cuda")
        self.temperature = torch.full((T,), 3.0, device="cuda")
        self.Q = torch.zeros(T, dec.V, device="cuda")
        self.fill(seed)

    def fill(self, seed):
        g = torch.Generator().manual_seed(seed)
        T = len(self.token)
        tree = sum((some_tree(self.nodes, seed + i, 0.0) for i in range(self.dec.n)), [])
        self.parent.copy_(i32(tree))
        self.token.copy_(torch.randint(0, self.dec.V, (T,), generator=g).int())
        self.u.copy_(torch.rand(T, generator=g) * 0.05)
        self.u_next.copy_(torch.rand(self.dec.n, generator=g))
        self.Q.copy_(torch.softmax(torch.randn(T, self.dec.V, generator=g), 1))

    def __call__(self):
        return self.dec.step(self.token, self.parent, self.q_start, self.nodes, self.temperature, self.u, self.u_next,
                             Q=self.Q)


def test_kept_tokens_leave_the_cache_of_plain_appends():
    """Steps that begin with the token drawn last and keep some drafts: every cached row, bit for bit, as a
    decoder has it that gets the same tokens one by one; and each token's attention, read a step later as part of
    the sequence, is what a plain decoder computes."""
    r = random.Random(3)
    prompt = [[r.randrange(1003) for _ in range(29)] for _ in range(3)]
    fast, plain = Decoder(11), Decoder(11)
    nxt = fast.prompt(prompt)
    plain.prompt(prompt)
    s = Step(fast, 0, nodes=12)
    tokens, sizes = [[] for _ in range(3)], set()
    for k in range(25):
        s.fill(900 + 13 * k)
        s.token[::12] = nxt
        path, count, nxt = s()
        for i, (p, c) in enumerate(zip(path.tolist(), count.tolist())):
            tokens[i] += [int(s.token[12 * i + j]) for j in p[:c]]
            sizes.add(c)
    assert fast.length.tolist() == [29 + len(t) for t in tokens] and len(sizes) >= 3
    for k in range(max(map(len, tokens))):
        on = [k < len(t) for t in tokens]
        qs = [0]
        for o in on:
            qs.append(qs[-1] + o)
        plain.cache.append(*plain.split(i32([t[k] for t, o in zip(tokens, on) if o])), plain.table, plain.length, i32(qs), 1,
                           rope=plain.rope)
        plain.length += i32([int(o) for o in on])
    assert torch.equal(plain.length, fast.length)
    for a, b in zip(rows_of(plain), rows_of(fast)):
        assert torch.equal(a, b)
    # both go on alike
    x = i32([5, 6, 7])
    assert torch.equal(plain.one(x), fast.one(x))


def state_of(dec):
    c = dec.cache
    return [t.clone() for t in (dec.length, c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.k_window, c.v_window)]


def test_a_step_in_a_graph():
    """A captured step follows the trees, lengths and numbers of each replay; two graphs of two decoders, and
    eager steps between the replays."""
    decs = [Decoder(5), Decoder(5), Decoder(5)]
    steps = [Step(d, 1) for d in decs]
    r = random.Random(1)
    prompt = [[r.randrange(1003) for _ in range(40)] for _ in range(3)]
    for d in decs:
        d.prompt(prompt)
    torch.cuda.synchronize()
    eager = steps[0]
    warm = [state_of(d) for d in decs]
    for s in steps:
        s()
    graphs, outs = [], []
    for s in steps[1:]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s())
        graphs.append(g)
    for d, w in zip(decs, warm):                             # back to where the prompt left it
        for t, v in zip((d.length, d.cache.k_codes, d.cache.v_codes, d.cache.k_scale, d.cache.v_scale,
                         d.cache.k_window, d.cache.v_window), w):
            t.copy_(v)
    kept = 0
    for k in range(30):
        for s in steps:
            s.fill(100 + 7 * k)
        want = eager()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), k
        for d in decs[1:]:
            for a, b in zip(state_of(d), state_of(decs[0])):
                assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float())), k
        kept += int(want[1].sum())
    assert kept > 3 * 30                                    # some drafts were kept


def test_steps_on_other_streams():
    """On a stream given by argument, on current side streams, two decoders at once: the same as alone."""
    r = random.Random(2)
    prompt = [[r.randrange(1003) for _ in range(50)] for _ in range(3)]
    decs = [Decoder(6) for _ in range(3)]
    steps = [Step(d, 1) for d in decs]
    for d in decs:
        d.prompt(prompt)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(12):
        for s in steps:
            s.fill(500 + 11 * k)
        torch.cuda.synchronize()
        got = []
        for s, st in zip(steps[1:], streams):
            with torch.cuda.stream(st):
                got.append(s())
        want = steps[0]()
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want))
    st, s, d = streams[0], steps[0], decs[0]
    args = (d.table, d.length, s.q_start, s.nodes)
    x = d.split(s.token)
    torch.cuda.synchronize()
    q = d.cache.append_tree(*x, *args, s.parent, rope=d.rope, stream=st)
    o, lse = d.cache.attend_tree(q, *args, s.parent, want_lse=True, stream=st)
    st.synchronize()
    assert torch.equal(q, d.cache.append_tree(*x, *args, s.parent, rope=d.rope))
    o2, lse2 = d.cache.attend_tree(q, *args, s.parent, want_lse=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    P = oq.token_probs(d.logits(o))
    torch.cuda.synchronize()
    assert torch.equal(oq.token_probs(d.logits(o), stream=st), P)
    a = oq.tree_verify(s.token, s.parent, s.q_start, s.nodes, P, s.u, s.u_next, Q=s.Q, stream=st)
    st.synchronize()
    b = oq.tree_verify(s.token, s.parent, s.q_start, s.nodes, P, s.u, s.u_next, Q=s.Q)
    assert all(torch.equal(i, j) for i, j in zip(a, b))
    d.cache.commit(*a[:2], *args, stream=st)
    st.synchronize()
    before = state_of(d)
    d.cache.commit(i32([[0]] * 3), i32([0] * 3), *args)
    for i, j in zip(before, state_of(d)):
        assert torch.equal(torch.nan_to_num(i.float()), torch.nan_to_num(j.float()))


def test_calls_repeat_bit_for_bit():
    b = Trees(5, 16, 2, 128, 64, 2500, seed=4, s_a=False)
    b.step([2000, 3, 700, 64, 1500], attend=False)
    parents = [some_tree(n, n) for n in (40, 1, 64, 7, 20)]
    qkv = b.new([len(p) for p in parents]).cuda()
    args = (b.table, i32(b.len), i32(b.starts([len(p) for p in parents])), 64)
    par = i32(sum(parents, []))
    w = 16 * 128
    outs = []
    for _ in range(4):
        q = b.cache.append_tree(qkv[:, :w], qkv[:, w:w + 256], qkv[:, w + 256:], *args, par, rope=b.rope, slots=b.slots)
        outs.append((q, *b.cache.attend_tree(q, *args, par, slots=b.slots, want_lse=True)))
    for o in outs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(o, outs[0]))


def test_a_step_dropped():
    """A tree that is not committed leaves nothing behind: the next step is as if it had not been."""
    a, b = (Trees(2, 4, 2, 64, 32, 400, seed=9) for _ in range(2))
    for t in (a, b):
        t.step([100, 31], attend=False)
    junk = [some_tree(32, 1), chain(32)]
    state = a.g.get_state()
    a.tree_step(junk, [[], []], attend=False)
    a.g.set_state(state)
    for t in (a, b):
        t.tree_step([some_tree(9, 5), chain(3)], [[0], [0, 1, 2]])
        t.step([40, 1])
        t.check_rows()
    assert torch.equal(a.cache.k_codes, b.cache.k_codes) and torch.equal(a.cache.v_scale.nan_to_num(), b.cache.v_scale.nan_to_num())


@pytest.mark.parametrize("H,Hkv,n", [(80, 1, 3), (130, 2, 7), (256, 2, 1)])
def test_more_heads_to_a_group_than_a_tile_has_rows(H, Hkv, n):
    b = Trees(2, H, Hkv, 64, 32, 300, seed=H, s_a=False, rope=False)
    b.step([200, 45], attend=False)
    b.tree_step([some_tree(n, 1), some_tree(max(1, n - 2), 2)], [[0], []])
