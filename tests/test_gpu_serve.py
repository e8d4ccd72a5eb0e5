"""The serving operators of a weight-activation quantised block against plain
64-bit references: RMSNorm to codes, the 8-bit integer linear, the paged 8-bit
cache and attention over it."""
import pytest
import torch

from paper_2308_13137_amd import oq
from tests import serve_ref as ref
from tests.serve_ref import BF8, F24, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand(seed, *shape, scale=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


# ------------------------------------------------------------------ RMSNorm to codes
NORM = [(1, 8, BF, BF), (3, 64, F32, None), (1, 4096, BF, BF), (5, 5120, F32, BF), (2, 2056, BF, F32),
        (7, 11008, BF, None), (2, 16384, F32, F32), (1, 32768, BF, BF), (300, 1032, BF, BF),
        (3, 8200, F32, BF), (1100, 256, F32, F32),
        (2500, 1032, BF, F32), (2049, 2048, F32, BF), (9, 6144, BF, BF)]


@pytest.mark.parametrize("T,D,xt,rt", NORM)
@pytest.mark.parametrize("shift", [False, True])
def test_norm_values(T, D, xt, rt, shift):
    X = rand(1, T, D, scale=3.0, dtype=xt)
    R = None if rt is None else rand(2, T, D, dtype=rt)
    gain, bias = rand(3, D) + 1.0, rand(4, D) if shift else None
    H, y, codes, h, z = oq.rmsnorm_quant(X, gain, 16, R=R, bias=bias, eps=1e-5, dq_dtype=F32)
    assert codes is None and h is None and z is None
    rH, ry, ry0 = ref.norm64(X, R, gain, bias, 1e-5)
    assert torch.equal(H.cpu(), rH)
    # rstd, its product with H, the product with the gain: half a step each; then the shift's sum
    tol = 3.1 * F24 * ry0.abs() + 1.1 * F24 * ry.abs()
    assert ((f64(y) - ry).abs() <= tol).all()


@pytest.mark.parametrize("T,D,xt,rt", NORM)
@pytest.mark.parametrize("bits", [8, 4, 6 | oq.ACT_SYM, 2])
def test_norm_codes_are_the_quantisers(T, D, xt, rt, bits):
    """Codes, steps and zero points equal those of act_fakequant_fwd on the fp32 norm, bit for bit;
    the fused addition equals an addition first."""
    X = rand(5, T, D, scale=2.0, dtype=xt)
    R = None if rt is None else rand(6, T, D, dtype=rt)
    gain, bias = rand(7, D) + 1.0, rand(8, D, scale=0.1)
    H, dq, codes, h, z = oq.rmsnorm_quant(X, gain, bits, R=R, bias=bias, dq_dtype=F32)
    _, y, _, _, _ = oq.rmsnorm_quant(H, gain, 16, bias=bias, dq_dtype=F32)
    rdq, rcodes, rh, rz = oq.act_fakequant_fwd(y, bits)
    for a, b in ((codes, rcodes), (h, rh), (z, rz), (dq, rdq)):
        assert torch.equal(a, b)
    _, dq16, c2, h2, _ = oq.rmsnorm_quant(H, gain, bits, bias=bias, dq_dtype=BF)
    assert torch.equal(c2, codes) and torch.equal(h2, h) and torch.equal(dq16, rdq.to(BF))


def test_norm_in_place_and_bare():
    X, R, gain = rand(1, 33, 512, dtype=BF), rand(2, 33, 512, dtype=BF), rand(3, 512)
    want = oq.rmsnorm_quant(X, gain, 8, R=R)
    for alias in ("X", "R"):
        x, r = X.clone(), R.clone()
        H, dq, codes, h, z = oq.rmsnorm_quant(x, gain, 8, R=r, H=x if alias == "X" else r)
        assert H.data_ptr() == (x if alias == "X" else r).data_ptr() and dq is None
        assert torch.equal(H, want[0]) and torch.equal(codes, want[2]) and torch.equal(h, want[3])
    H, dq, codes, h, z = oq.rmsnorm_quant(X, gain, 8, codes=False, hz=False)
    assert H is X and (dq, codes, h, z) == (None,) * 4
    assert oq.rmsnorm_quant(X[:0], gain, 8)[2].shape == (0, 512)


def test_norm_extremes():
    """Rows of zeros, of the type's largest values and with values that are not finite."""
    D, gain = 256, torch.ones(256, device="cuda")
    big = torch.finfo(BF).max
    X = torch.stack([torch.zeros(D), torch.full((D,), big), torch.full((D,), 1e-30), torch.ones(D),
                     torch.ones(D), torch.ones(D)]).to(BF)
    X[1, ::2] = -big
    X[3, 5], X[4, 200], X[5, 255] = float("nan"), float("inf"), -float("inf")
    H, dq, codes, h, z = oq.rmsnorm_quant(X.cuda(), gain, 8, dq_dtype=F32)
    h, dq, codes, z = h.cpu(), dq.cpu(), codes.cpu(), z.cpu()
    assert h[0] == h[2] and float(h[0]) == float(torch.tensor(1e-5)) and (dq[0] == 0).all()
    # the largest values have a mean square in fp64: the row is +-1
    assert torch.isfinite(h[1]) and (dq[1].abs() - 1).abs().max() <= h[1] / 2 * 1.001
    for r in (3, 4, 5):
        assert torch.isnan(h[r]) and (codes[r] == 0).all() and z[r] == 0 and torch.isnan(dq[r]).all()


# ------------------------------------------------------------------ the 8-bit linear
def linear_case(seed, T, K, N, top=255, zspread=30.0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, top + 1, (T, K), generator=g).to(torch.uint8)
    w = torch.randint(0, top + 1, (N, K), generator=g).to(torch.uint8)
    z = torch.round(top / 2 + zspread * torch.randn(T, generator=g))
    zw = torch.round(top / 2 + zspread * torch.randn(N, generator=g))
    h, hw = torch.rand(T, generator=g) + 0.1, torch.rand(N, generator=g) * 0.01 + 1e-4
    B = torch.randn(N, generator=g)
    return [t.cuda() for t in (codes, h, z, w, hw, zw, B)]


def check_linear(T, K, N, out=F32, bias=True, seed=0, top=255, zspread=30.0):
    codes, h, z, w, hw, zw, B = linear_case(seed, T, K, N, top, zspread)
    B = B if bias else None
    packed, wsum = oq.int8_pack(w)
    y = oq.int8_linear(codes, h, z, packed, wsum, hw, zw, B=B, out_dtype=out)
    r = ref.linear64(codes, h, z, w, hw, zw, None)
    full = r if B is None else r + f64(B)
    # the integer sum rounded to fp32, h_x h_w, their product, the sum with the bias; the output's type
    tol = 3.01 * F24 * r.abs() + 1.01 * F24 * full.abs() + (1.01 * BF8 * full.abs() if out == BF else 0)
    assert y.dtype == out and ((f64(y) - full).abs() <= tol).all()
    return y


LIN = [(1, 16, 1), (1, 4096, 4096), (2, 80, 16), (3, 48, 40), (5, 5120, 264), (16, 256, 17), (17, 1040, 100),
       (33, 4112, 130), (64, 512, 8), (65, 192, 250), (100, 1008, 264), (127, 320, 511), (128, 128, 128),
       (130, 2064, 770), (257, 512, 1000), (300, 144, 4100), (515, 4096, 520)]


@pytest.mark.parametrize("T,K,N", LIN)
@pytest.mark.parametrize("out", [F32, BF])
def test_linear(T, K, N, out):
    check_linear(T, K, N, out, bias=T % 2 == 1, seed=T + K + N)


# one size for each tile of the kernels' rule, with row and channel counts that end inside a tile
TILES = [(9, 3001), (17, 100), (31, 9002), (64, 9001), (61, 20003), (128, 20008), (131, 20002), (300, 30001)]


@pytest.mark.parametrize("T,N", TILES)
@pytest.mark.parametrize("K", [16, 64, 144, 208, 1040, 2064])
def test_linear_every_tile(T, N, K):
    """Inner sizes from less than one k-step to several ring turns, whole and ragged."""
    check_linear(T, K, N, BF if K == 208 else F32, bias=K == 144, seed=K)


@pytest.mark.parametrize("T,K", [(200, 1040), (193, 2064), (256, 48)])
def test_linear_several_token_tiles(T, K):
    check_linear(T, K, 8190, BF, bias=True, seed=T)


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("top,zspread", [(3, 0.0), (15, 5.0), (63, 1000.0), (255, 30000.0)])
def test_linear_widths_and_far_zero_points(T, top, zspread):
    check_linear(T, 528, 144, F32, top=top, zspread=zspread, seed=top)


@pytest.mark.parametrize("T,N", [(1, 32), (20, 32), (256, 32), (20, 9000), (60, 20000), (300, 30000)])
def test_linear_extreme_codes(T, N):
    """All codes 0 against all 255 at the largest width: the sum is the largest that can be."""
    K = 65536
    for a, b in ((0, 0), (255, 255), (0, 255)):
        codes = torch.full((T, K), a, dtype=torch.uint8, device="cuda")
        w = torch.full((N, K), b, dtype=torch.uint8, device="cuda")
        one, zero = torch.ones(T, device="cuda"), torch.full((T,), 128.0, device="cuda")
        ones, zeros = torch.ones(N, device="cuda"), torch.full((N,), 128.0, device="cuda")
        packed, wsum = oq.int8_pack(w)
        assert (wsum == K * (b - 128)).all()
        y = oq.int8_linear(codes, one, zero, packed, wsum, ones, zeros)
        want = float(K * (a - 128) * (b - 128))
        assert (y.double() - want).abs().max() <= F24 * abs(want)


def test_linear_rows_do_not_depend_on_the_batch():
    codes, h, z, w, hw, zw, B = linear_case(9, 700, 528, 9000)
    packed, wsum = oq.int8_pack(w)
    full = oq.int8_linear(codes, h, z, packed, wsum, hw, zw, B=B)
    for a, b in ((0, 1), (0, 16), (0, 30), (0, 37), (64, 164), (0, 300)):
        part = oq.int8_linear(codes[a:b].contiguous(), h[a:b].clone(), z[a:b].clone(), packed, wsum, hw, zw, B=B)
        assert torch.equal(part, full[a:b])


def test_linear_takes_the_quantisers_outputs():
    """act_fakequant_fwd's and lwc_fakequant_fwd's codes as they come, against their dequantised product."""
    X, W = rand(1, 50, 512, dtype=BF), rand(2, 96, 512, scale=0.05, dtype=BF)
    lg = torch.full((96, 1), 4.0, device="cuda")
    Xd, cx, hx, zx = oq.act_fakequant_fwd(X, 6, dq_dtype=F32)
    Wd, cw, hw, zw = oq.lwc_fakequant_fwd(W, lg, lg, 4, 512, dq_dtype=F32)
    packed, wsum = oq.int8_pack(cw)
    y = oq.int8_linear(cx, hx, zx, packed, wsum, hw, zw)
    r = ref.linear64(cx, hx, zx, cw, hw, zw, None)
    assert ((f64(y) - r).abs() <= 3.01 * F24 * r.abs()).all()
    # the dequantised factors round once each
    d = f64(Xd) @ f64(Wd).t()
    assert ((f64(y) - d).abs() <= 4.01 * F24 * (f64(Xd).abs() @ f64(Wd).abs().t())).all()


def test_linear_pack_layout_and_empty():
    g = torch.Generator().manual_seed(3)
    w = torch.randint(0, 256, (21, 80), generator=g).to(torch.uint8)
    packed, wsum = oq.int8_pack(w.cuda())
    b = torch.zeros(32, 128, dtype=torch.int16)
    b[:21, :80] = w.to(torch.int16) - 128
    want = b.view(2, 16, 2, 4, 16).permute(0, 2, 3, 1, 4).to(torch.int8)
    assert torch.equal(packed.cpu(), want) and torch.equal(wsum.cpu(), b[:21].to(torch.int32).sum(1).to(torch.int32))
    codes, h, z, w, hw, zw, B = linear_case(1, 4, 32, 8)
    packed, wsum = oq.int8_pack(w)
    assert oq.int8_linear(codes[:0], h[:0], z[:0], packed, wsum, hw, zw).shape == (0, 8)


# ------------------------------------------------------------------ the cache
def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Batch:
    """A cache with plain copies of every sequence beside it."""

    def __init__(self, n_seq, H, Hkv, d, page, max_tokens, seed=0, rope=True, s_a=True, dtype=BF):
        self.n, self.H, self.Hkv, self.d, self.P, self.dtype = n_seq, H, Hkv, d, page, dtype
        self.g = torch.Generator().manual_seed(seed)
        mp = -(-max_tokens // page)
        self.cache = oq.KVCache(n_seq * mp + 2, page, Hkv, d, n_seq + 1)
        # what was in the memory before must not matter
        self.cache.k_window.fill_(float("nan"))
        self.cache.v_window.fill_(float("inf"))
        self.cache.k_scale.fill_(float("nan"))
        self.cache.v_scale.fill_(float("nan"))
        self.table = torch.randperm(n_seq * mp, generator=self.g).to(torch.int32).view(n_seq, mp).cuda()
        self.slots = i32([n_seq - i for i in range(n_seq)])
        self.rope = oq.rope_table(max_tokens, d) if rope else None
        self.s_a = (torch.rand(Hkv * d, generator=self.g) + 0.5).cuda() if s_a else None
        self.k = [ref.PlainCache(page, Hkv, d) for _ in range(n_seq)]
        self.v = [ref.PlainCache(page, Hkv, d) for _ in range(n_seq)]
        self.len = [0] * n_seq

    def new(self, counts):
        T, W = sum(counts), (self.H + 2 * self.Hkv) * self.d
        return torch.randn(T, W, generator=self.g).to(self.dtype)

    def plain(self, qkv, counts):
        """Q~ of the new tokens in the kernel's fp32 order; K~ and V join the plain copies."""
        H, Hkv, d = self.H, self.Hkv, self.d
        pos = torch.cat([torch.arange(L, L + c) for L, c in zip(self.len, counts)])
        x = qkv.float().view(len(qkv), H + 2 * Hkv, d)
        q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
        if self.rope is not None:
            cs, sn = (self.rope.cpu()[pos][:, None, :, j] for j in (0, 1))
            q, k = ref.turn32(q, cs, sn), ref.turn32(k, cs, sn)
        if self.s_a is not None:
            sa = self.s_a.cpu().view(Hkv, d)
            q, k = q / sa.repeat_interleave(H // Hkv, 0), k * sa
        at = 0
        for i, c in enumerate(counts):
            self.k[i].add(k[at:at + c].to(BF))
            self.v[i].add(v[at:at + c].to(BF))
            at += c
        return q.to(BF)

    def starts(self, counts):
        s = [0]
        for c in counts:
            s.append(s[-1] + c)
        return s

    def step(self, counts, attend=True, pad=3, max_q=None):
        """append + attend of `counts` new tokens, checked; `pad` rows behind the last sequence."""
        H, Hkv, d = self.H, self.Hkv, self.d
        qkv = self.new(counts)
        T = len(qkv)
        full = torch.cat([qkv, torch.full((pad, qkv.shape[1]), float("nan")).to(self.dtype)]).cuda()
        length, qs, mq = i32(self.len), i32(self.starts(counts)), max_q or max(counts)
        want_q = self.plain(qkv, counts)
        out = torch.full((T + pad, H * d), 7.0, dtype=BF, device="cuda")
        q = self.cache.append(full[:, :H * d], full[:, H * d:(H + Hkv) * d], full[:, (H + Hkv) * d:], self.table,
                              length, qs, mq, rope=self.rope, s_a=self.s_a, slots=self.slots, out=out)
        assert q is out and torch.equal(q[:T].cpu().view(T, H, d), want_q) and (q[T:] == 7).all()
        if attend:
            o = torch.full((T + pad, H * d), 7.0, dtype=BF, device="cuda")
            _, lse = self.cache.attend(q, self.table, length, qs, mq, slots=self.slots, want_lse=True, out=o)
            assert (o[T:] == 7).all()
            at = 0
            for i, c in enumerate(counts):
                if c:
                    r, tol, rl = ref.attend64(want_q[at:at + c], self.k[i].values(), self.v[i].values(), self.len[i])
                    err = (f64(o[at:at + c]).view(c, H, d) - r).abs()
                    assert (err <= tol).all(), (i, float((err / tol).max()))
                    assert ((f64(lse)[:, at:at + c] - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()
                at += c
        self.len = [a + c for a, c in zip(self.len, counts)]

    def check_rows(self):
        """Every cached row, full pages and the open one, bit for bit."""
        rs = self.starts(self.len)
        zero = i32([0] * self.n)
        k, v = self.cache.read(self.table, zero, i32(self.len), i32([0] * (self.n + 1)), i32(rs), rs[-1],
                               max(self.len), slots=self.slots, dtype=F32)
        for got, plain in ((k, self.k), (v, self.v)):
            want = torch.cat([p.values() for p in plain]).reshape(rs[-1], -1)
            assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2), (5, 1)])
def test_cache_steps(d, page, H, Hkv):
    """Prompts, then decoding, then chunks that end pages in every position."""
    b = Batch(3, H, Hkv, d, page, 700, seed=d + page + H)
    for counts in ([150, 1, 33], [1, 1, 1], [0, 31, 1], [3, 0, 63], [1, 129, 200], [page, 2 * page, 1]):
        b.step(counts)
    b.check_rows()


@pytest.mark.parametrize("dtype,rope,s_a", [(F32, True, True), (F32, True, False), (BF, False, False),
                                            (F32, False, True)])
def test_cache_inputs(dtype, rope, s_a):
    b = Batch(2, 4, 2, 128, 64, 400, seed=5, rope=rope, s_a=s_a, dtype=dtype)
    for counts in ([100, 7], [1, 57], [64, 64]):
        b.step(counts)
    b.check_rows()


def test_cache_codes_do_not_depend_on_the_chunks():
    """One prompt call, single tokens and odd chunks leave the same codes, steps and windows."""
    d, P, n = 128, 32, 150
    qkv = rand(1, n, 6 * d, dtype=BF)
    rope = oq.rope_table(256, d)
    got = []
    for chunks in ([n], [1] * n, [37, 90, 23], [31, 1, 33, 85]):
        c = oq.KVCache(8, P, 2, d, 1)
        L = 0
        for m in chunks:
            x = qkv[L:L + m]
            c.append(x[:, :2 * d], x[:, 2 * d:4 * d], x[:, 4 * d:], i32([[5, 0, 2, 7, 1, 3, 4, 6]]), i32([L]),
                     i32([0, m]), m, rope=rope)
            L += m
        # the open page's half and the one before it
        half, rows = (n // P) % 2, n % P
        got.append([c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.k_window[0, half, :, :rows * d],
                    c.k_window[0, 1 - half], c.v_window[0, 1 - half]])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("back", [1, 17, 32, 50])
def test_cache_drops_the_newest_tokens(back):
    """Lowering `length` within the last two pages and appending others equals never having had them."""
    d, P = 64, 32
    b = Batch(1, 2, 2, d, P, 400, seed=back)
    b.step([115])
    b.step([9])
    b.len[0] -= back
    for p in b.k + b.v:
        p.rows = p.rows[:b.len[0]]
    b.step([70])
    b.check_rows()


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 40])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (16, 2), (40, 8)])
def test_attend_rows(n, H, Hkv):
    """Row counts around the row tiles, behind a prefix."""
    b = Batch(2, H, Hkv, 64, 32, 200, seed=n + H, s_a=False)
    b.step([70, 95], attend=False)
    b.step([n, 1 + n // 2])


@pytest.mark.parametrize("L", [1, 31, 32, 33, 1000, 4095, 4096])
def test_attend_long_single_token(L):
    b = Batch(1, 4, 2, 128, 64, 4200, seed=L, s_a=False)
    b.step([L], attend=False)
    b.step([1])


def test_attend_ragged_lengths_split():
    """Short and long sequences in one batch: some splits have no tokens."""
    b = Batch(5, 4, 1, 64, 64, 3000, seed=3)
    b.step([1, 2900, 40, 64, 700], attend=False)
    b.step([1, 1, 1, 1, 1])


def test_attend_large_scores():
    """Scores of hundreds: the softmax is nearly one-hot and nothing overflows."""
    b = Batch(1, 2, 2, 64, 32, 300, seed=11, rope=False, s_a=False)
    b.new = lambda counts: 40.0 * torch.randn(sum(counts), 6 * 64, generator=b.g).to(BF)
    b.step([120])
    b.step([1])


def test_attend_values_that_are_not_finite():
    """A row that sees a NaN or an infinity is NaN, the rows before it are exact."""
    for kind in ("k", "v"):
        for bad in (float("nan"), float("inf"), -float("inf")):
            for at in (40, 70):                     # in a page that fills up; in the open page
                b = Batch(1, 2, 1, 64, 32, 200, seed=1, rope=False, s_a=False)
                qkv = b.new([80])
                clean = qkv.clone()
                col = (2 if kind == "k" else 3) * 64 + 5
                qkv[at, col] = bad
                outs = []
                for x in (qkv, clean):
                    x = x.cuda()
                    args = (b.table, i32([0]), i32([0, 80]), 80)
                    q = b.cache.append(x[:, :128], x[:, 128:192], x[:, 192:], *args)
                    outs.append(b.cache.attend(q, *args))
                first = at if at >= 64 else at // 32 * 32     # a full page stands for NaN as a whole
                got = outs[0].float()
                assert torch.isfinite(got[:first]).all() and torch.isnan(got[at:]).all(), (kind, bad, at)
                if at >= 64:
                    assert torch.equal(outs[0][:first], outs[1][:first])


def test_cache_entries_that_do_not_fit():
    """Sequences with bad pages, slots, lengths or row ranges: NaN rows, nothing written, others untouched."""
    d, P, n = 64, 32, 6
    cache = oq.KVCache(12, P, 1, d, n)
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(6, 2)
    table[1, 0], table[2, 0] = -1, 12
    x = rand(1, 6 * 40, 3 * d, dtype=BF)
    slots = i32([0, 1, 2, -1, 6, 5])
    length = i32([0, 0, 0, 0, 0, 30])              # the last one passes the table's two pages
    qs = i32([0, 40, 80, 120, 160, 200, 240])
    before = [t.clone() for t in (cache.k_codes, cache.k_scale, cache.k_window, cache.v_window)]
    q = cache.append(x[:, :d], x[:, d:2 * d], x[:, 2 * d:], table, length, qs, 40, slots=slots)
    o = cache.attend(q, table, length, qs, 40, slots=slots)
    torch.cuda.synchronize()
    assert torch.isfinite(q[:120].float()).all() and torch.isnan(q[120:].float()).all()
    assert torch.isfinite(o[:40].float()).all() and torch.isnan(o[40:].float()).all()
    assert torch.equal(cache.k_codes[1:], before[0][1:]) and torch.equal(cache.k_scale[1:], before[1][1:])
    assert torch.equal(cache.k_window[3:], before[2][3:]) and torch.equal(cache.v_window[3:], before[3][3:])
    # row ranges outside the batch's rows
    for starts in ([0, 40, 300], [-1, 40, 80], [0, 50, 40], [0, 41, 60]):
        o = torch.full((80, d), 7.0, dtype=BF, device="cuda")
        cache.attend(q[:80].contiguous(), table[:2], length[:2], i32(starts), 40, out=o)
        torch.cuda.synchronize()


def test_shared_pages():
    """Two sequences with the same full pages and their own windows read the same rows."""
    d, P = 128, 64
    b = Batch(2, 2, 2, d, P, 256, seed=4)
    qkv = b.new([130])
    for i in range(2):
        x = qkv.cuda()
        b.cache.append(x[:, :2 * d], x[:, 2 * d:4 * d], x[:, 4 * d:], b.table[:1], i32([0]), i32([0, 130]), 130,
                       rope=b.rope, slots=i32([i]))
    table = torch.stack([b.table[0], b.table[0]])
    q = rand(9, 2, 2 * d, dtype=BF)
    q[1] = q[0]
    o = b.cache.attend(q, table, i32([129, 129]), i32([0, 1, 2]), 1, slots=i32([0, 1]))
    assert torch.equal(o[0], o[1]) and torch.isfinite(o.float()).all()


@pytest.mark.parametrize("H,Hkv,page", [(4, 1, 128), (20, 4, 128), (40, 8, 32)])
def test_cache_few_heads(H, Hkv, page):
    """Chunks that end pages, at few key heads with many query heads, beside single tokens and empty ones."""
    b = Batch(4, H, Hkv, 128, page, 400, seed=H)
    b.step([142, 0, 77, 1])
    b.step([1, 5, 130, 0])
    b.check_rows()


@pytest.mark.parametrize("d,long", [(64, (66,)), (128, (0, 69)), (64, (3, 30, 31))])
def test_cache_ragged_batch(d, long):
    """Prompts among 70 sequences that decode or rest, more than one wave's worth."""
    b = Batch(70, 8, 8, d, 32, 2200, seed=d + len(long))
    b.step([1 + 7 * (i % 9) for i in range(70)], attend=False)
    counts = [int(i % 5 != 1) for i in range(70)]
    for i in long:
        counts[i] = 300 + i
    b.step(counts)
    b.step([1] * 70)
    b.check_rows()


def test_cache_ragged_batch_grouped():
    """Row tiles of grouped heads that begin inside a token, few rows of one sequence beside many of another."""
    b = Batch(66, 40, 8, 64, 64, 700, seed=8, s_a=False)
    b.step([600 - 8 * i if i < 60 else 0 for i in range(66)], attend=False)
    b.step([1] * 20 + [7] * 20 + [0] * 10 + [40] + [2] * 14 + [90])


def test_ragged_entries_that_do_not_fit():
    """In a batch whose units are searched for: bad sequences are NaN (the first max_q rows of a range that is
    longer), the others as without them."""
    d, P, n, Hkv = 64, 32, 70, 8
    counts = [1] * n
    counts[5], counts[6], counts[40], counts[65], counts[66] = 200, 90, 200, 200, 70
    qs = [0]
    for k in counts:
        qs.append(qs[-1] + k)
    T = qs[-1]
    x = rand(2, T, 3 * Hkv * d, dtype=BF)
    rows = torch.arange(T, device="cuda")

    def run(bad):
        cache = oq.KVCache(n * 8, P, Hkv, d, n)
        table = torch.arange(n * 8, dtype=torch.int32, device="cuda").view(n, 8)
        slots, length, mq = list(range(n)), [3] * n, 200
        if bad:
            slots[5], length[65], table[40, 1], mq = n, 8 * P - 100, n * 8, 199
        w = Hkv * d
        args = (table, i32(length), i32(qs), mq)
        q = torch.full((T, w), 7.0, dtype=BF, device="cuda")
        cache.append(x[:, :w], x[:, w:2 * w], x[:, 2 * w:], *args, slots=i32(slots), out=q)
        o = torch.full((T, w), 7.0, dtype=BF, device="cuda")
        cache.attend(q, *args, slots=i32(slots), out=o)
        return q, o

    (q0, o0), (q1, o1) = run(False), run(True)
    assert torch.isfinite(q0.float()).all() and torch.isfinite(o0.float()).all()
    lost = torch.zeros(T, dtype=torch.bool, device="cuda")
    for i in (5, 40, 65):                           # longer than max_q now, all three
        a, e = qs[i], qs[i] + 199
        lost |= (rows >= a) & (rows <= e)
        assert torch.isnan(q1[a:e].float()).all() and torch.isnan(o1[a:e].float()).all()
        assert (q1[e] == 7).all() and (o1[e] == 7).all()
    assert torch.equal(q1[~lost], q0[~lost]) and torch.equal(o1[~lost], o0[~lost])


def test_outputs_in_place():
    """The queries turned in their own rows, the output over the queries."""
    for counts in ([130, 1, 33], [1, 1, 1]):
        H, Hkv, d, P = 16, 2, 128, 64
        T, W = sum(counts), H * d
        table = torch.arange(18, dtype=torch.int32, device="cuda").view(3, 6)
        qs = i32([0, counts[0], counts[0] + counts[1], T])
        q, k, v = rand(3, T, W, dtype=BF), rand(4, T, Hkv * d, dtype=BF), rand(5, T, Hkv * d, dtype=BF)
        rope, s_a = oq.rope_table(400, d), rand(6, Hkv * d).abs() + 0.5
        got = []
        for place in (False, True):
            c = oq.KVCache(18, P, Hkv, d, 3)
            args = (table, i32([9, 200, 0]), qs, max(counts))
            x = q.clone()
            t = c.append(x, k, v, *args, rope=rope, s_a=s_a, out=x if place else None)
            c.k_scale.fill_(0.01)
            c.v_scale.fill_(0.01)
            got.append((t.clone(), c.attend(t, *args, out=t if place else None)))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_cache_offsets_past_32_bits():
    """Pages and windows that begin more than 4 GiB into their tensors."""
    H = Hkv = 8
    d, P = 128, 128
    n_pages, n_slots = 2 ** 32 // (Hkv * P * d) + 64, 2 ** 32 // (2 * Hkv * P * d * 2) + 64
    cache = oq.KVCache(n_pages, P, Hkv, d, n_slots)
    assert cache.k_codes.numel() > 2 ** 32 and cache.k_window.numel() * 2 > 2 ** 32
    small = oq.KVCache(3, P, Hkv, d, 1)
    T, w = 300, Hkv * d
    x = rand(7, T + 1, 3 * w, dtype=BF)
    out = []
    for c, pages, slot in ((cache, [n_pages - 1, n_pages - 40, n_pages - 2], n_slots - 1), (small, [0, 1, 2], 0)):
        table = i32([pages])
        for at, n in ((0, T), (T, 1)):
            r = x[at:at + n]
            args = (table, i32([at]), i32([0, n]), n)
            q = c.append(r[:, :w], r[:, w:2 * w], r[:, 2 * w:], *args, slots=i32([slot]))
            out.append(c.attend(q, *args, slots=i32([slot])))
        k, v = c.read(table, i32([0]), i32([T]), i32([0, 1]), i32([0, T + 1]), T + 1, T + 1, slots=i32([slot]))
        out += [k, v]
    for a, b in zip(out[:4], out[4:]):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b)


def test_rows_past_32_bits():
    """The last rows of tensors of more than 2^31 elements."""
    T, D, N = 270000, 64, 8192                      # codes [T, D], products [T, N]
    codes = torch.randint(0, 256, (T, D), dtype=torch.uint8, device="cuda")
    h, z = torch.full((T,), 0.01, device="cuda"), torch.full((T,), 128.0, device="cuda")
    wc = torch.randint(0, 256, (N, D), dtype=torch.uint8, device="cuda")
    hw, zw = torch.full((N,), 0.01, device="cuda"), torch.full((N,), 127.0, device="cuda")
    packed, wsum = oq.int8_pack(wc)
    y = oq.int8_linear(codes, h, z, packed, wsum, hw, zw, out_dtype=BF)
    assert y.numel() > 2 ** 31
    tail = slice(T - 300, T)
    assert torch.equal(y[tail], oq.int8_linear(codes[tail].clone(), h[tail].clone(), z[tail].clone(), packed, wsum,
                                               hw, zw, out_dtype=BF))
    gain = torch.ones(N, device="cuda")
    _, _, c, hh, zz = oq.rmsnorm_quant(y, gain, 8)
    _, _, c1, h1, z1 = oq.rmsnorm_quant(y[tail].clone(), gain, 8)
    assert torch.equal(c[tail], c1) and torch.equal(hh[tail], h1) and torch.equal(zz[tail], z1)


def test_cache_drops_twice():
    """Dropped, filled a little and dropped again, never below the page before the furthest."""
    d, P = 64, 32
    b = Batch(1, 2, 2, d, P, 400, seed=12)
    b.step([124])
    for to, new in ((70, 5), (64, 3), (66, 40), (97, 1), (96, 33)):
        b.len[0] = to
        for p in b.k + b.v:
            p.rows = p.rows[:to]
        b.step([new])
        b.check_rows()


@pytest.mark.parametrize("before,counts,H,Hkv", [
    ([300, 0, 130, 64], [200, 333, 1, 70], 2, 2),             # levels that several sequences share
    ([0, 640, 5], [129, 257, 0], 10, 2),                      # an empty one; tiles that begin inside a token
    ([1000, 0], [150, 140], 1, 1),                            # no level in common
    ([33 * (i % 7) for i in range(32)], [40 + 13 * (i % 11) for i in range(32)], 4, 1),
])
def test_attend_longest_first(before, counts, H, Hkv):
    b = Batch(len(counts), H, Hkv, 64, 32, 1400, seed=len(counts), s_a=False)
    if any(before):
        b.step(before, attend=False)
    b.step(counts)


def test_longest_first_entries_that_do_not_fit():
    """A chunk longer than the table's pages, a length beyond them: NaN, the others as without them."""
    d, P, H = 64, 32, 2
    counts = [200, 150, 300, 170]
    qs = [0, 200, 350, 650, 820]
    x = rand(8, 820, 3 * H * d, dtype=BF)

    def run(bad):
        cache = oq.KVCache(32, P, H, d, 4)
        table = torch.arange(32, dtype=torch.int32, device="cuda").view(4, 8)
        length = i32([0, 2 ** 31 - 1 if bad else 9, 0, 50])   # the third one's 300 tokens pass 8 pages of 32
        args = (table, length, i32(qs), 300)
        w = H * d
        q = cache.append(x[:, :w], x[:, w:2 * w], x[:, 2 * w:], *args)
        return q, cache.attend(q, *args)

    (q0, o0), (q1, o1) = run(False), run(True)
    for q, o in ((q0, o0), (q1, o1)):
        assert torch.isnan(q[350:650].float()).all() and torch.isnan(o[350:650].float()).all()
        assert torch.isfinite(o[:200].float()).all() and torch.isfinite(o[650:].float()).all()
    assert torch.isfinite(o0[200:350].float()).all() and torch.isnan(o1[200:350].float()).all()
    keep = [*range(200), *range(650, 820)]
    assert torch.equal(o0[keep], o1[keep])


@pytest.mark.parametrize("n,H", [(1, 2), (3, 2), (70, 1), (150, 2)])
def test_attend_pages_never_written(n, H):
    """Zeroed pages before the new tokens: keys and values of zero."""
    d, P, L = 64, 32, 96
    cache = oq.KVCache(8, P, 1, d, 1)
    x = rand(n, n, (H + 2) * d, dtype=BF)
    args = (torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8), i32([L]), i32([0, n]), n)
    q = cache.append(x[:, :H * d], x[:, H * d:(H + 1) * d], x[:, (H + 1) * d:], *args)
    o = cache.attend(q, *args)
    k, v = ref.PlainCache(P, 1, d), ref.PlainCache(P, 1, d)
    for c, at in ((k, H), (v, H + 1)):
        c.add(torch.cat([torch.zeros(L, d, dtype=BF), x[:, at * d:(at + 1) * d].cpu()]).view(L + n, 1, d))
    r, tol, _ = ref.attend64(q.cpu().view(n, H, d), k.values(), v.values(), L)
    assert ((f64(o).view(n, H, d) - r).abs() <= tol).all()


@pytest.mark.parametrize("n,H,before", [(1, 4, 200), (7, 2, 40), (40, 2, 70), (150, 2, 33), (150, 2, 0)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_attend_queries_that_are_not_finite(n, H, before, bad):
    """One head's query with a value that is not finite: that row is NaN, the others are as without it."""
    d, P = 64, 32
    cache = oq.KVCache(8, P, 1, d, 1)
    x = rand(before, before + n, (H + 2) * d, dtype=BF)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    for at, m in ((0, before), (before, n)):
        if m:
            r = x[at:at + m]
            args = (table, i32([at]), i32([0, m]), m)
            q = cache.append(r[:, :H * d], r[:, H * d:(H + 1) * d], r[:, (H + 1) * d:], *args)
    clean = cache.attend(q, *args).view(n, H, d)
    row, head = n // 2, H - 1
    q.view(n, H, d)[row, head, 11] = bad
    got = cache.attend(q, *args).view(n, H, d)
    assert torch.isnan(got[row, head].float()).all()
    keep = torch.ones(n, H, dtype=torch.bool, device="cuda")
    keep[row, head] = False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("d,H,Hkv,before,counts", [(128, 4, 4, [0], [400]), (64, 8, 2, [0, 70], [129, 33]),
                                                   (128, 10, 2, [30], [65]), (64, 1, 1, [1100, 1], [90, 200])])
def test_attend_short_prompts(d, H, Hkv, before, counts):
    """Prompts too few to fill the card in tiles of 128 rows."""
    b = Batch(len(counts), H, Hkv, d, 64, 1300, seed=d + H, s_a=False)
    if any(before):
        b.step(before, attend=False)
    b.step(counts)
