"""Drafted tokens against the target: probabilities from logits, and the walk that keeps part of
a tree, against plain 64-bit references."""
import random

import pytest
import torch

from paper_2308_13137_amd import oq
from tests import tree_ref
from tests.test_gpu_serve import i32, rand
from tests.test_gpu_tree import chain, some_tree, star

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------ probabilities
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 1000, 4099, 32000, 50257, 65536, 128256, 131073, 300001])
@pytest.mark.parametrize("dt", [BF, F32])
def test_probs(V, dt):
    T = 3 if V > 60000 else 37
    x = rand(V, T, V, scale=3.0, dtype=dt)
    if V > 8:
        x[0, 1::3] = -float("inf")
    t = (0.3 + torch.rand(T, generator=torch.Generator().manual_seed(V))).cuda()
    for temp in (None, t):
        got = oq.token_probs(x, temp)
        want, tol = tree_ref.probs64(x, temp)
        assert got.dtype == F32 and ((got.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("V", [5, 1000, 32003, 128256, 200001])
@pytest.mark.parametrize("dt", [BF, F32])
def test_probs_at_temperature_zero(V, dt):
    """One at the first of the largest logits, ties among them in every part of a row."""
    T = 16
    x = rand(V, T, V, dtype=dt)
    g = torch.Generator().manual_seed(1)
    for t in range(T):
        x[t, torch.randint(0, V, (4,), generator=g)] = 50.0
    x[1, V - 1] = 60.0
    x[2, 0] = x[2, V - 1] = 70.0
    got = oq.token_probs(x, torch.zeros(T, device="cuda")).cpu()
    first = torch.stack([(r == r.max()).nonzero()[0, 0] for r in x.cpu().float()])
    assert torch.equal(got, torch.nn.functional.one_hot(first, V).float())


@pytest.mark.parametrize("V", [8191, 8192, 16383, 16385, 70001, 128256, 200003])
@pytest.mark.parametrize("dt", [BF, F32])
def test_probs_of_few_rows_are_those_of_many(V, dt):
    """Rows that several workgroups share have the bits of rows that one has, whatever their kind, and
    nothing beside them is written."""
    many = rand(V, 130, V, scale=3.0, dtype=dt)
    many[1, V - 1], many[2, :], many[3, V // 2] = float("nan"), -float("inf"), 90.0
    t = torch.ones(130, device="cuda")
    t[3], t[4], t[5], t[6] = 0.0, 0.0, -1.0, 0.4
    want = oq.token_probs(many, t)
    for T in (1, 7, 33, 70):
        out = torch.full((T + 1, V + 5), 7.0, device="cuda")
        oq.token_probs(many[:T], t[:T], out=out[:T, 3:3 + V])
        assert torch.equal(out[:T, 3:3 + V].view(torch.int32), want[:T].view(torch.int32)), T
        assert (out[:T, :3] == 7).all() and (out[:T, 3 + V:] == 7).all() and (out[T] == 7).all()


def test_probs_strides_and_rows_that_are_none():
    V = 1003
    wide = rand(1, 12, 2000, dtype=BF)
    x = wide[:, 5:5 + V]
    out = torch.full((12, 1200), 7.0, device="cuda")
    assert torch.equal(oq.token_probs(x, out=out[:, 3:3 + V]), oq.token_probs(x.contiguous()))
    assert (out[:, :3] == 7).all() and (out[:, 3 + V:] == 7).all()
    assert oq.token_probs(x[:0]).shape == (0, V)
    for V in (64, 1003, 140000):
        for dt in (BF, F32):
            x = rand(2, 9, V, dtype=dt)
            x[0, V - 1], x[1, 3], x[2, :] = float("nan"), float("inf"), -float("inf")
            x[3, 1:] = -float("inf")
            t = torch.tensor([1, 1, 1, 0.5, -1, float("nan"), float("inf"), 1e-42, 1.0], device="cuda")
            got = oq.token_probs(x, t).cpu()
            for r in (0, 1, 2, 4, 5, 6):
                assert torch.isnan(got[r]).all(), (V, r)
            assert got[3, 0] == 1 and (got[3, 1:] == 0).all()
            assert got[7, x[7].float().argmax()] == 1 and got[7].sum() == 1
            got0 = oq.token_probs(x, torch.zeros(9, device="cuda")).cpu()
            assert torch.isnan(got0[:3]).all() and (got0[3:].sum(1) == 1).all()


def test_probs_extremes():
    """The type's ends, and temperatures from tiny to huge."""
    big = torch.finfo(F32).max
    x = torch.tensor([[big, -big, 0.0, big], [1e-30, -1e-30, 0.0, 2e-30], [88.0, 89.0, -200.0, 0.0]], device="cuda")
    got = oq.token_probs(x).cpu()
    assert torch.equal(got[0], torch.tensor([0.5, 0.0, 0.0, 0.5]))
    assert torch.allclose(got[1], torch.full((4,), 0.25), rtol=0, atol=2.0 ** -23)
    for temp in (1e-3, 30.0, 1e30):
        t = torch.full((1,), temp, device="cuda")
        want, tol = tree_ref.probs64(x[2:], t)
        assert ((oq.token_probs(x[2:], t).cpu().double() - want).abs() <= tol).all()


def test_probs_past_32_bits():
    T, V = 16400, 131072                                     # 2^31 elements and more
    assert T * V > 2 ** 31
    x = torch.zeros(T, V, dtype=BF, device="cuda")
    x[-1] = rand(1, 1, V, dtype=BF)[0]
    got = oq.token_probs(x)
    assert torch.equal(got[-1:], oq.token_probs(x[-1:].clone())) and (got[-2] == 1.0 / V).all() and (got[0] == 1.0 / V).all()


# ------------------------------------------------------------------ verification
def verify_case(seed, n_seq, max_n, V, mode, spread=1.5, tree=None):
    g = torch.Generator().manual_seed(seed)
    r = random.Random(seed)
    trees = [tree or some_tree(r.randint(1, max_n) if i else max_n, seed + i, 0.03) for i in range(n_seq)]
    start = [0]
    for t in trees:
        start.append(start[-1] + len(t))
    T = start[-1]
    x = torch.randn(T, V, generator=g) * spread
    P = torch.softmax(x, 1)
    Q = torch.softmax(x + 0.8 * torch.randn(T, V, generator=g), 1)
    token = torch.zeros(T, dtype=torch.int32)
    for b, t in zip(start, trees):
        for c in range(len(t)):
            kids = [j for j, p in enumerate(t) if p == c]
            if not kids:
                continue
            if mode == "certain":
                take = torch.topk(Q[b + c], min(V, len(kids))).indices.tolist()
            elif mode == "distinct":
                take = torch.multinomial(Q[b + c], min(V, len(kids)), generator=g).tolist()
            else:
                take = torch.multinomial(Q[b + c], len(kids), replacement=True, generator=g).tolist()
            for k, j in enumerate(kids):
                token[b + j] = take[k % len(take)]
    u, un = torch.rand(T, generator=g), torch.rand(n_seq, generator=g)
    return trees, start, token, P, (None if mode == "certain" else Q), u, un


def check_verify(trees, start, token, P, Q, u, un, replace, max_q=None, **kw):
    mq = max_q or max(len(t) for t in trees)
    cuda = [None if t is None else t.cuda() for t in (token, P, u, un, Q)]
    path, count, nxt = oq.tree_verify(cuda[0], i32(sum(trees, [])), i32(start), mq, cuda[1], cuda[2], cuda[3], Q=cuda[4],
                                      replace=replace, **kw)
    path, count, nxt = path.cpu().tolist(), count.cpu().tolist(), nxt.cpu().tolist()
    kept = 0
    for i, (b, t) in enumerate(zip(start, trees)):
        e = b + len(t)
        want = ([], -1) if not t else tree_ref.verify64(token[b:e].tolist(), t, P[b:e], None if Q is None else Q[b:e],
                                                        u[b:e].tolist(), un[i], replace)
        assert path[i] == want[0] + [-1] * (mq - len(want[0])) and count[i] == len(want[0]), (i, path[i], want)
        assert nxt[i] == want[1], (i, nxt[i], want)
        kept += count[i]
    return kept


@pytest.mark.parametrize("mode", ["draws", "distinct", "certain"])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 64, 257, 1000, 5003, 40000])
def test_verify(mode, V):
    for seed in range(3):
        case = verify_case(seed, 12, 40 if V < 10000 else 14, V, mode)
        check_verify(*case, replace=mode != "distinct")


@pytest.mark.parametrize("mode", ["draws", "distinct", "certain"])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128])
def test_verify_tree_sizes(mode, n):
    case = verify_case(n, 6, n, 97, mode, spread=0.5)
    check_verify(*case, replace=mode != "distinct", max_q=n + (n < 128))
    # chains that are kept to the end: the draft is the target
    trees, start, token, P, Q, u, un = verify_case(n, 4, n, 97, mode, tree=chain(n))
    if Q is not None:
        assert check_verify(trees, start, token, Q, Q, u * 0.999, un, replace=mode != "distinct") == 4 * n


@pytest.mark.parametrize("mode", ["draws", "distinct"])
def test_verify_many_siblings(mode):
    """Stars whose children are all rejected but few: long chains of residuals."""
    trees, start, token, P, Q, u, un = verify_case(4, 8, 100, 700, mode, tree=star(100))
    u = 0.9 + 0.1 * u
    check_verify(trees, start, token, P, Q, u, un, replace=mode != "distinct")
    # and a draft that is far off: the residual is the target until its token comes
    far = torch.softmax(torch.randn(len(P), 700, generator=torch.Generator().manual_seed(1)) * 4, 1)
    check_verify(trees, start, token, P, far, u, un, replace=mode != "distinct")


@pytest.mark.parametrize("mode", ["draws", "distinct"])
def test_verify_peaked_drafts(mode):
    """Nearly all of q in one token, whose siblings come from the little that is left."""
    V, tree = 300, star(6)
    for seed in range(5):
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(6, V, generator=g)
        P = torch.softmax(x, 1)
        y = x.clone()
        y[:, 7] += 17.0
        Q = torch.softmax(y, 1)
        token = torch.tensor([0, 7] + torch.multinomial(P[0], 4, generator=g).tolist(), dtype=torch.int32)
        u, un = torch.rand(6, generator=g), torch.rand(1, generator=g)
        check_verify([tree], [0, 6], token, P, Q, u, un, replace=mode != "distinct")


def test_verify_borders():
    """Numbers that are exact: ties between u q and p reject, a running sum that equals the draw passes it."""
    V = 8
    P = torch.tensor([[1, 2, 1, 0, 0, 2, 1, 1.0]]).repeat(2, 1) / 8
    Q = torch.tensor([[4, 1, 1, 1, 0, 1, 0, 0.0]]).repeat(2, 1) / 8
    for token, u, kept in ((0, 0.25, False), (0, 0.2499, True), (1, 0.99, True), (3, 0.0, False), (4, 0.0, False),
                           (6, 0.99, True)):
        tok, uu = torch.tensor([0, token], dtype=torch.int32), torch.tensor([0.0, u])
        for un in (0.0, 0.125, 0.375, 0.4999, 0.5, 0.75, 0.875, 1 - 2.0 ** -24):
            check_verify([[-1, 0]], [0, 2], tok, P, Q, uu, torch.tensor([un]), replace=True)
        path, count, nxt = oq.tree_verify(tok.cuda(), i32([-1, 0]), i32([0, 2]), 2, P.cuda(), uu.cuda(),
                                          torch.tensor([0.5], device="cuda"), Q=Q.cuda())
        assert count.item() == 1 + kept
        if kept:                                             # p itself: 1/8 2/8 1/8 | the running sum is 1/2 there
            assert nxt.item() == 5


def test_verify_residuals_without_mass():
    """A draft that covers the target: after a rejection (by rounding, or a u of one) nothing is left, and the draw is
    from the distribution before it."""
    P = torch.tensor([[0.5, 0.5, 0.0, 0.0]]).repeat(4, 1)
    Q = P.clone()
    for replace in (True, False):
        for tree, tok in (([-1, 0], [0, 0]), ([-1, 0, 0], [0, 0, 1]), ([-1, 0, 0, 0], [0, 1, 0, 1])):
            n = len(tree)
            check_verify([tree], [0, n], torch.tensor(tok, dtype=torch.int32), P[:n], Q[:n], torch.ones(n),
                         torch.tensor([0.7]), replace=replace)
    one = torch.tensor([[0.0, 1.0, 0.0, 0.0]]).repeat(3, 1)
    check_verify([[-1, 0, 0]], [0, 3], torch.tensor([0, 1, 2], dtype=torch.int32), one, None, torch.ones(3),
                 torch.tensor([0.7]), replace=True)


def test_verify_greedy():
    """Temperature zero: the path follows the target's largest logits, the next token is the last one's."""
    V, tree = 1000, [-1, 0, 0, 1, 1, 2, 3]
    x = rand(3, 7, V)
    P = oq.token_probs(x, torch.zeros(7, device="cuda"))
    top = x.argmax(1).cpu().tolist()
    token = torch.tensor([5, top[0], 9, 11, top[1], 3, 2], dtype=torch.int32)
    path, count, nxt = oq.tree_verify(token.cuda(), i32(tree), i32([0, 7]), 7, P, torch.rand(7, device="cuda"),
                                      torch.rand(1, device="cuda"))
    assert path.tolist() == [[0, 1, 4, -1, -1, -1, -1]] and count.item() == 3 and nxt.item() == top[4]


@pytest.mark.parametrize("mode", ["draws", "distinct", "certain"])
def test_verify_keeps_the_targets_distribution(mode):
    """60,000 drafts of one tree: the first and the second new token come as often as the target has
    them (five standard deviations of a count)."""
    n, V, tree = 60000, 6, [-1, 0, 0, 0, 1]
    m = len(tree)
    g = torch.Generator().manual_seed(7)
    P1 = torch.softmax(1.2 * torch.randn(m, V, generator=g), 1)
    Q1 = torch.softmax(1.2 * torch.randn(m, V, generator=g), 1)
    token = torch.zeros(n, m, dtype=torch.int32)
    if mode == "draws":
        token[:, 1:4] = torch.multinomial(Q1[0], 3 * n, replacement=True, generator=g).view(n, 3).int()
    elif mode == "distinct":
        token[:, 1:4] = torch.multinomial(Q1[:1].expand(n, V), 3, generator=g).int()
    else:
        token[:, 1:4] = torch.topk(Q1[0], 3).indices.int()
    token[:, 4] = torch.multinomial(Q1[1], n, replacement=True, generator=g).int()
    P, Q = P1.repeat(n, 1).cuda(), None if mode == "certain" else Q1.repeat(n, 1).cuda()
    u, un = torch.rand(n * m, generator=g).cuda(), torch.rand(n, generator=g).cuda()
    path, count, nxt = oq.tree_verify(token.view(-1).cuda(), i32(tree * n), i32([m * i for i in range(n + 1)]), m, P, u,
                                      un, Q=Q, replace=mode != "distinct")
    path, count, nxt = path.cpu().long(), count.cpu(), nxt.cpu().long()
    assert (nxt >= 0).all() and (count >= 1).all() and (count <= 3).all()
    at1 = token.gather(1, path[:, 1:2].clamp(min=0))[:, 0].long()
    first = torch.where(count > 1, at1, nxt)

    def fits(tokens, p):
        k = len(tokens)
        freq = torch.bincount(tokens, minlength=V).double() / k
        p = p.double()
        return ((freq - p).abs() <= 5 * (p * (1 - p) / k).sqrt() + 1e-6).all()
    assert fits(first, P1[0])
    # behind node 1 (with a child) and nodes 2, 3 (without): the second new token
    for node in (1, 2, 3):
        here = (count > 1) & (path[:, 1] == node)
        at2 = token.gather(1, path[:, 2:3].clamp(min=0))[:, 0].long()
        second = torch.where(count > 2, at2, nxt)[here]
        if len(second) > 200:
            assert fits(second, P1[node]), node


def test_verify_rows_that_are_none():
    """Bad rows, parents, tokens and probabilities; other trees are untouched."""
    V, n = 500, 8
    trees, start, token, P, Q, u, un = verify_case(1, 9, n, V, "draws", tree=star(n))
    want = None
    for bad in (False, True):
        p, q, tok, par, qs = P.clone(), Q.clone(), token.clone(), sum(trees, []), list(start)
        if bad:
            p[start[1]] = float("nan")
            p[start[2], 7] = float("inf")
            p[start[3]] = 0.0
            par[start[4] + 5] = 5
            par[start[5] + 2] = -7
            tok[start[6] + 1:start[6] + n] = torch.tensor([-1, V, 2 ** 31 - 1, -2 ** 31, V + 5, -9, V])
            qs[9] = start[9] + 1                             # rows past the tensor
        got = [t.cpu() for t in oq.tree_verify(tok.cuda(), i32(par), i32(qs), n, p.cuda(), torch.full((len(u),), 0.99).cuda(),
                                               un.cuda(), Q=q.cuda())]
        if not bad:
            want = got
            continue
        path, count, nxt = got
        assert nxt[[1, 3, 4, 5, 8]].tolist() == [-1] * 5
        # beside an infinity a child may be kept, and its own row is fine
        b, e = start[2], start[3]
        kept = tree_ref.verify64(tok[b:e].tolist(), trees[2], p[b:e], q[b:e], torch.full((n,), 0.99).tolist(), un[2], True)
        assert (path[2, :count[2]].tolist(), nxt[2]) == kept
        assert count[[4, 5, 8]].tolist() == [0] * 3 and (path[[4, 5, 8]] == -1).all()
        # tokens that are none are rejected, and the draw is from the target
        assert count[6] == 1 and nxt[6] == tree_ref.verify64([0], [-1], P[start[6]:], None, [0], un[6], True)[1]
        for i in (0, 7):
            for a, b in zip(got, want):
                assert torch.equal(a[i], b[i])
    # a draw from the target's own row does not look at the draft's
    q = torch.full_like(Q, float("nan"))
    leaf = oq.tree_verify(token[:1].cuda(), i32([-1]), i32([0, 1]), 1, P[:1].cuda(), u[:1].cuda(), un[:1].cuda(), Q=q[:1].cuda())
    assert leaf[2].item() == tree_ref.verify64([0], [-1], P[:1], None, [0], un[0], True)[1]
    # trees without nodes; parents that hang on the sequence are never kept
    empty = oq.tree_verify(token.cuda(), i32(sum(trees, [])), i32([0, 0, 8]), 8, P.cuda(), u.cuda(), un[:2].cuda())
    assert empty[1][0] == 0 and empty[2][0] == -1 and (empty[0][0] == -1).all() and empty[1][1] >= 1
    lone = oq.tree_verify(token[:3].cuda(), i32([-1, -1, -1]), i32([0, 3]), 3, P[:3].cuda(), u[:3].cuda() * 0,
                          un[:1].cuda())
    assert lone[0].tolist() == [[0, -1, -1]]


def test_verify_strided_rows():
    trees, start, token, P, Q, u, un = verify_case(5, 5, 20, 333, "draws")
    wide = torch.full((len(P), 1000), float("nan"), device="cuda")
    wide[:, 11:344], wide[:, 500:833] = P.cuda(), Q.cuda()
    par, qs = i32(sum(trees, [])), i32(start)
    a = oq.tree_verify(token.cuda(), par, qs, 20, wide[:, 11:344], u.cuda(), un.cuda(), Q=wide[:, 500:833])
    b = oq.tree_verify(token.cuda(), par, qs, 20, P.cuda(), u.cuda(), un.cuda(), Q=Q.cuda())
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refusals_on_the_gpu():
    x = torch.zeros(4, 50, device="cuda")
    i, f = i32([0, 0, 0, 0]), torch.zeros(4, device="cuda")
    par, qs, un = i32([-1, 0, 0, 1]), i32([0, 4]), torch.zeros(1, device="cuda")
    oq.tree_verify(i, par, qs, 4, x, f, un, Q=x)
    for a, kw in (((i.long(), par, qs, 4, x, f, un), {}), ((i, par[:3], qs, 4, x, f, un), {}), ((i, par, qs[:1], 4, x, f, un), {}),
                  ((i, par, qs, 4, x.bfloat16(), f, un), {}), ((i, par, qs, 4, x, f[:2], un), {}),
                  ((i, par, qs, 4, x, f, un), dict(Q=x[:3])), ((i, par, qs, 4, x, f, un), dict(Q=x[:, :49])),
                  ((i, par, qs, 4, x.t().contiguous().t(), f, un), {}), ((i, par, qs.cpu(), 4, x, f, un), {}),
                  ((i, par, qs, 200, x.repeat(60, 1), f, un), {})):
        with pytest.raises(oq.OQError):
            oq.tree_verify(*a, **kw)
    for call in (lambda: oq.token_probs(x.half()), lambda: oq.token_probs(x, f[:3]), lambda: oq.token_probs(x, out=x),
                 lambda: oq.token_probs(x, out=x.bfloat16()), lambda: oq.token_probs(x[:, :0]),
                 lambda: oq.token_probs(torch.zeros(1, 2 ** 20 + 1, device="cuda"))):
        with pytest.raises(oq.OQError):
            call()
    c = oq.KVCache(4, 32, 1, 64, 1)
    q, kv = torch.zeros(2, 64, dtype=BF, device="cuda"), torch.zeros(2, 64, dtype=BF, device="cuda")
    args = (i32([[0, 1]]), i32([0]), i32([0, 2]))
    c.append_tree(q, kv, kv, *args, 2, i32([-1, 0]))
    big = torch.zeros(40, 64, dtype=BF, device="cuda")
    for call in (lambda: c.append_tree(q, kv, kv, *args, 2, i32([-1])), lambda: c.append_tree(q, kv, kv, *args, 2, i32([-1, 0]).long()),
                 lambda: c.append_tree(q, kv, kv, *args, 2, i32([-1, 0]).cpu()),
                 lambda: c.append_tree(big, big, big, *args, 40, i32(chain(40))),
                 lambda: c.attend_tree(big, *args, 40, i32(chain(40))), lambda: c.attend_tree(q.float(), *args, 2, i32([-1, 0])),
                 lambda: c.commit(i32([[0]]), i32([1, 1]), *args, 2), lambda: c.commit(i32([[0]]).long(), i32([1]), *args, 2),
                 lambda: c.commit(i32([[0]]), i32([1]), *args, 33)):
        with pytest.raises(oq.OQError):
            call()
