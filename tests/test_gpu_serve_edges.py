"""Calls at the edges of what the serving operators' header allows."""
import pytest
import torch

from paper_2308_13137_amd import oq
from tests import serve_ref as ref
from tests.serve_ref import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rand(seed, *shape, scale=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def split(x, H, Hkv, d):
    return x[:, :H * d], x[:, H * d:(H + Hkv) * d], x[:, (H + Hkv) * d:]


# (new tokens, query heads of one key head): 16 and 32 rows of a workgroup, tiles of 64 rows (the first of
# them with a full page and the open one in a tile) and of 128
ROWS = [(1, 2), (3, 2), (9, 2), (5, 8), (70, 1), (150, 2)]


# ------------------------------------------------------------------ steps of zero
@pytest.mark.parametrize("n,H", ROWS)
@pytest.mark.parametrize("which", ["k", "v", "kv"])
def test_zero_steps_stand_for_zeros_whatever_the_codes(n, H, which):
    """Pages whose steps are zero but whose codes are not (a pool's recycled pages): attention as over the
    rows that KVCache.read returns, which are zeros."""
    d, P, L = 64, 32, 96
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    args = (table, i32([L]), i32([0, n]), n)
    x = rand(n, n, (H + 2) * d, dtype=BF)
    x[:, :H * d] *= 16.0
    c = oq.KVCache(8, P, 1, d, 1)
    g = torch.Generator().manual_seed(7)
    for name, codes, step in (("k", c.k_codes, c.k_scale), ("v", c.v_codes, c.v_scale)):
        codes.copy_(torch.randint(-127, 128, codes.shape, generator=g).to(torch.int8))
        step.fill_(0.02)
        if name in which:
            step[:3] = 0.0
    q = c.append(*split(x, H, 1, d), *args)
    o, lse = c.attend(q, *args, want_lse=True)
    k, v = c.read(table, i32([0]), i32([L]), i32([0, n]), i32([0, L + n]), L + n, L + n, dtype=F32)
    for name, t in (("k", k), ("v", v)):
        assert (t[:L] == 0).all() == (name in which)
    r, tol, rl = ref.attend64(q.cpu().view(n, H, d), k.cpu().view(-1, 1, d), v.cpu().view(-1, 1, d), L)
    assert ((f64(o).view(n, H, d) - r).abs() <= tol).all()
    assert ((f64(lse) - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()


# ------------------------------------------------------------------ values of very different sizes
@pytest.mark.parametrize("n,H", ROWS)
@pytest.mark.parametrize("big", [2.0 ** 60, 2.0 ** 90, 2.0 ** 96, 2.0 ** 118])
@pytest.mark.parametrize("small", [0.0, 1e-4, 1.0])
def test_value_steps_far_apart(n, H, big, small):
    """One page of very large values, whose keys point away from every query, beside pages of small ones or
    pages never written: every token counts in the log-sum-exp, and the output keeps the header's bound."""
    d, P, L = 64, 32, 288
    table = torch.arange(15, dtype=torch.int32, device="cuda").view(1, 15)
    x = rand(n + H, L + n, (H + 2) * d, dtype=BF)
    x[:, :H * d] *= 3.0
    x[:, (H + 1) * d:] *= small if small else 1e-4
    for at in range(0, H * d, d):
        x[:, at] = 8.0
    x[:, H * d] = 0.0
    x[32:64, H * d] = -16.0                          # their scores are 16 lower
    x[32:64, (H + 1) * d:] = rand(3, 32, d).clamp(-2, 2).mul(big / 2).to(BF)
    c = oq.KVCache(15, P, 1, d, 1)
    if small:
        c.append(*split(x[:L], H, 1, d), table, i32([0]), i32([0, L]), L)
    else:                                            # (the others' codes and steps stay zero)
        c.append(*split(x[32:64], H, 1, d), table[:, 1:].contiguous(), i32([0]), i32([0, 32]), 32)
    args = (table, i32([L]), i32([0, n]), n)
    q = c.append(*split(x[L:], H, 1, d), *args)
    o, lse = c.attend(q, *args, want_lse=True)
    k, v = c.read(table, i32([0]), i32([L]), i32([0, n]), i32([0, L + n]), L + n, L + n, dtype=F32)
    r, tol, rl = ref.attend64(q.cpu().view(n, H, d), k.cpu().view(-1, 1, d), v.cpu().view(-1, 1, d), L)
    assert ((f64(lse) - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()
    assert ((f64(o).view(n, H, d) - r).abs() <= tol).all()


# ------------------------------------------------------------------ rows that are NaN
@pytest.mark.parametrize("n,H,L", [(1, 2, 96), (1, 2, 2100), (9, 2, 96), (70, 1, 96), (70, 1, 2100), (150, 2, 33)])
def test_log_sum_exp_of_a_row_that_is_nan(n, H, L):
    """An infinite query against keys of one sign: every score is -inf, output and log-sum-exp are NaN."""
    d, P = 64, 32
    pages = -(-(L + n) // P)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    x = rand(n, L + n, (H + 2) * d, dtype=BF)
    x[:, H * d + 5] = 1.0
    c = oq.KVCache(pages, P, 1, d, 1)
    c.append(*split(x[:L], H, 1, d), table, i32([0]), i32([0, L]), L)
    args = (table, i32([L]), i32([0, n]), n)
    q = c.append(*split(x[L:], H, 1, d), *args)
    clean, clean_lse = c.attend(q, *args, want_lse=True)
    q.view(n, H, d)[n // 2, H - 1, 5] = -float("inf")
    o, lse = c.attend(q, *args, want_lse=True)
    bad = torch.zeros(n, H, dtype=torch.bool, device="cuda")
    bad[n // 2, H - 1] = True
    assert torch.isnan(o.view(n, H, d)[bad].float()).all() and torch.isnan(lse.t()[bad]).all()
    assert torch.equal(o.view(n, H, d)[~bad], clean.view(n, H, d)[~bad])
    assert torch.equal(lse.t()[~bad], clean_lse.t()[~bad])


# ------------------------------------------------------------------ bounds far above the batch
@pytest.mark.parametrize("most", [70, 1 << 20, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, 1 << 40])
def test_read_with_a_bound_far_above_the_rows(most):
    """max_rows is at least the largest number of rows: any larger one gives the same."""
    d, P, n = 64, 32, 70
    c = oq.KVCache(3, P, 1, d, 1)
    x = rand(1, n, 3 * d, dtype=BF)
    table = i32([[2, 0, 1]])
    c.append(*split(x, 1, 1, d), table, i32([0]), i32([0, n]), n)
    torch.full((2, n, d), 7.0, dtype=BF, device="cuda")      # (what an output's memory may hold)
    k, v = c.read(table, i32([0]), i32([n]), i32([0, 0]), i32([0, n]), n, most)
    k1, v1 = c.read(table, i32([0]), i32([n]), i32([0, 0]), i32([0, n]), n, n)
    assert torch.equal(k, k1) and torch.equal(v, v1)
    assert torch.equal(k[64:], x[64:, d:2 * d]) and torch.equal(v[64:], x[64:, 2 * d:])


# ------------------------------------------------------------------ row ranges outside the batch
@pytest.mark.parametrize("H", [1, 4])
@pytest.mark.parametrize("starts,clean,ok,nan", [
    ([0, 40, 300], [0, 40, 80], [(0, 40)], [(40, 80)]),      # past the batch's rows: those inside are NaN
    ([-1, 40, 80], [0, 40, 80], [(40, 80)], [(0, 40)]),      # before them
    ([0, 50, 40], None, [], [(0, 40)]),                      # longer than max_q: its first max_q rows; decreasing
    ([0, 41, 60], [1, 41, 60], [(41, 60)], [(0, 40)]),
])
def test_row_ranges_outside_the_batch(H, starts, clean, ok, nan):
    """Such a sequence is not cached and its rows inside the batch are NaN, in the queries, the output and the
    log-sum-exp; its neighbour is as without it and rows of no sequence are left as they were."""
    d, P, T = 64, 32, 80
    x = rand(5, T, (H + 2) * d, dtype=BF)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)

    def run(qs):
        c = oq.KVCache(4, P, 1, d, 2)
        q, o = (torch.full((T, H * d), 7.0, dtype=BF, device="cuda") for _ in range(2))
        args = (table, i32([0, 0]), i32(qs), 40)
        c.append(*split(x, H, 1, d), *args, out=q)
        _, lse = c.attend(q, *args, want_lse=True, out=o)
        return c, q, o, lse.t()

    c, q, o, lse = run(starts)
    left = torch.ones(T, dtype=torch.bool)
    for a, b in nan:
        left[a:b] = False
        for t in (q, o, lse):
            assert torch.isnan(t[a:b].float()).all()
    for a, b in ok:
        left[a:b] = False
    assert (q[left] == 7).all() and (o[left] == 7).all()
    if clean is None:
        assert not c.k_window.any() and not c.v_window.any() and not c.k_scale.any() and not c.v_scale.any()
        return
    c1, q1, o1, lse1 = run(clean)
    for a, b in ok:
        for t, t1 in ((q, q1), (o, o1), (lse, lse1)):
            assert torch.isfinite(t[a:b].float()).all() and torch.equal(t[a:b], t1[a:b])
    good = 0 if ok[0][0] == 0 else 1
    for t, t1 in ((c.k_window, c1.k_window), (c.v_window, c1.v_window)):
        assert torch.equal(t[good], t1[good]) and not t[1 - good].any()
    for t, t1 in ((c.k_codes, c1.k_codes), (c.v_codes, c1.v_codes), (c.k_scale, c1.k_scale), (c.v_scale, c1.v_scale)):
        assert torch.equal(t[2 * good:2 * good + 2], t1[2 * good:2 * good + 2])
        assert not t[2 * (1 - good):2 * (1 - good) + 2].any()


# ------------------------------------------------------------------ few tokens, very many channels
@pytest.mark.parametrize("T", [1, 16, 17])
@pytest.mark.parametrize("K", [144, 1040])
@pytest.mark.parametrize("N", [40001, 65553, 70000])
def test_linear_few_tokens_over_very_many_channels(T, K, N):
    """Tiles of 128 and 256 tokens that hold few: all of a tile's other rows repeat the last one."""
    g = torch.Generator().manual_seed(T + K + N)
    codes = torch.randint(0, 256, (T, K), generator=g).to(torch.uint8).cuda()
    w = torch.randint(0, 256, (N, K), generator=g).to(torch.uint8).cuda()
    z, zw = (torch.round(127 + 30 * torch.randn(m, generator=g)).cuda() for m in (T, N))
    h, hw = (torch.rand(m, generator=g).cuda() * 0.01 + 1e-4 for m in (T, N))
    packed, wsum = oq.int8_pack(w)
    y = oq.int8_linear(codes, h, z, packed, wsum, hw, zw)
    r = ref.linear64(codes, h, z, w, hw, zw, None)
    # the integer sum rounded to fp32, h_x h_w, their product
    assert ((f64(y) - r).abs() <= 3.01 * ref.F24 * r.abs()).all()


# ------------------------------------------------------------------ very large scores
@pytest.mark.parametrize("n,H", ROWS)
@pytest.mark.parametrize("scale", [2.0 ** 8, 2.0 ** 12, 2.0 ** 20, 2.0 ** 40])
@pytest.mark.parametrize("mode", ["above", "below", "below, then zero"])
def test_scores_far_beyond_fp32s_integers(n, H, scale, mode):
    """Keys c scale e_0 with whole c up to 127 and queries +-scale e_0: codes and products are exact, tokens of
    the same c tie bit for bit and any other lies at least scale^2 / 8 below, so a row's output is the mean of
    the values at its largest score.  What remains of the error: fp16 weights, the fp32 sums and a bf16 rounding."""
    d, P, L = 64, 32, 288
    T = L + n
    g = torch.Generator().manual_seed(n + H)
    c = torch.randint(1, 128, (T,), generator=g).float()
    c[::P], c[7::P] = 127.0, 1.0
    if mode == "below, then zero":
        c[256:288] = 0.0
    x = rand(n, T, (H + 2) * d)
    x[:, :(H + 1) * d] = 0.0
    for at in range(0, H * d, d):
        x[:, at] = scale if mode == "above" else -scale
    x[:, H * d] = c.cuda() * scale
    x = x.to(BF)
    pages = -(-T // P)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    cache = oq.KVCache(pages, P, 1, d, 1)
    cache.append(*split(x[:L], H, 1, d), table, i32([0]), i32([0, L]), L)
    args = (table, i32([L]), i32([0, n]), n)
    q = cache.append(*split(x[L:], H, 1, d), *args)
    o, lse = cache.attend(q, *args, want_lse=True)
    k, v = cache.read(table, i32([0]), i32([L]), i32([0, n]), i32([0, T]), T, T, dtype=F32)
    assert torch.equal(k[:, 0].cpu(), c * scale) and not k[:, 1:].any()
    r, _, rl = ref.attend64(q.cpu().view(n, H, d), k.cpu().view(-1, 1, d), v.cpu().view(-1, 1, d), L)
    best = c if mode == "above" else -c
    for j in range(n):
        top = best[:L + j + 1] == best[:L + j + 1].max()
        w = v[:L + j + 1].cpu().double()[top]
        assert (r[j] - w.mean(0)).abs().max() < 1e-12
        tol = w.abs().mean(0) * (ref.F11 + 2 * T * ref.F24) * 1.01 + r[j].abs() * ref.BF8 * 1.01
        assert ((f64(o[j]).view(H, d) - r[j]).abs() <= tol).all()
    assert ((f64(lse) - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()


# ------------------------------------------------------------------ norms at the ends of fp32
@pytest.mark.parametrize("D", [64, 1032, 4096, 8200, 20480])
@pytest.mark.parametrize("dtype,scale", [(BF, 2.0 ** 127), (F32, 2.0 ** 127), (F32, 2.0 ** 120), (BF, 2.0 ** -130),
                                         (F32, 2.0 ** -126), (F32, 2.0 ** -140)])
def test_norm_of_the_largest_and_smallest_values(D, dtype, scale):
    """Rows whose 1 / rms is below fp32's normal numbers or above its largest: the same roundings as elsewhere
    (rstd, its product with H, the product with the gain: half a step each)."""
    g = torch.Generator().manual_seed(D)
    X = ((torch.rand(3, D, generator=g) * 2 - 1) * scale).to(dtype).cuda()
    X[1] = X[1] * 0.0
    X[1, ::7] = scale                                   # (few large values, many zeros)
    if scale == 2.0 ** 127:
        X[2] = torch.finfo(dtype).max * X[2].sign()
    gain = (torch.randn(D, generator=g) + 1.0).cuda()
    eps = 1e-5 if scale > 1 else 0.0
    _, y, _, _, _ = oq.rmsnorm_quant(X, gain, 16, eps=eps, dq_dtype=F32)
    _, ry, ry0 = ref.norm64(X, None, gain, None, eps)
    assert ((f64(y) - ry).abs() <= 3.1 * ref.F24 * ry0.abs()).all()
    _, _, codes, h, z = oq.rmsnorm_quant(X, gain, 8, eps=eps)
    _, rcodes, rh, rz = oq.act_fakequant_fwd(y, 8)
    assert torch.equal(codes, rcodes) and torch.equal(h, rh) and torch.equal(z, rz)


# ------------------------------------------------------------------ what a row does not see
@pytest.mark.parametrize("n,H", [(70, 1), (150, 2), (96, 8)])
@pytest.mark.parametrize("P", [32, 64])
@pytest.mark.parametrize("L", [0, 64, 96])
@pytest.mark.parametrize("big", [2.0 ** 12, 2.0 ** 30, 2.0 ** 60])
def test_later_values_do_not_touch_earlier_rows(n, H, P, L, big):
    """A prompt whose values become very large from some page on: the rows before it are as accurate as if it
    were not there."""
    d = 64
    x = rand(n + L, L + n, (H + 2) * d, dtype=BF)
    at = -(-(L + 32) // P) * P                       # the first row of the large page
    x[at:, (H + 1) * d:] *= big
    pages = -(-(L + n) // P)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    c = oq.KVCache(pages, P, 1, d, 1)
    if L:
        c.append(*split(x[:L], H, 1, d), table, i32([0]), i32([0, L]), L)
    args = (table, i32([L]), i32([0, n]), n)
    q = c.append(*split(x[L:], H, 1, d), *args)
    o, lse = c.attend(q, *args, want_lse=True)
    k, v = c.read(table, i32([0]), i32([L]), i32([0, n]), i32([0, L + n]), L + n, L + n, dtype=F32)
    m = at - L                                       # rows that do not see it
    r, tol, rl = ref.attend64(q[:m].cpu().view(m, H, d), k[:at].cpu().view(-1, 1, d), v[:at].cpu().view(-1, 1, d), L)
    assert ((f64(o[:m]).view(m, H, d) - r).abs() <= tol).all()
    assert ((f64(lse[:, :m]) - rl).abs() <= 1e-4 + 1e-5 * rl.abs()).all()
