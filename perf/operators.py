"""Cases for the operators that serve a weight-activation quantised LLaMA block.

Four operators, in the order a deployed block runs them:

``norm``    H = X + R, RMSNorm of H, the result as integer codes with a step
            and a zero point per token (oq.rmsnorm_quant)
``linear``  the product of integer codes of activations and weights, scales
            and zero points per token and per channel (oq.int8_linear)
``append``  RoPE and the [Q, K] scale on a ragged batch's new tokens, which go
            into a paged cache: pages that fill up become 8-bit codes with one
            scale per page and head, the open page stays bf16
            (oq.KVCache.append; oq.KVCache.read returns the touched pages' rows)
``attend``  causal attention of a ragged batch's new tokens over that cache
            (oq.KVCache.attend)

With ``own`` false :func:`run` is elementary torch arithmetic in 32 bits.
"""
import itertools
import math
import random

import torch

own = False

DEV = "cuda"


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one decoded token between two linears of the 4096-wide block: latency
        dict(name="norm_token", op="norm", T=1, D=4096, x="bf16", r="bf16", bias=False, bits=8),
        # a ragged prompt batch at the 13B width, fp32 stream, LET's shift absorbed, 6-bit codes
        dict(name="norm_ragged_let", op="norm", T=731, D=5120, x="f32", r="bf16", bias=True, bits=6),
        # a long prompt at the 70B width: bandwidth
        dict(name="norm_prompt", op="norm", T=16384, D=8192, x="bf16", r="bf16", bias=True, bits=8),
        # one token through a 4096 x 4096 projection: the weight's bytes
        dict(name="linear_token", op="linear", T=1, K=4096, N=4096, y="f32", bias=True, bits=8),
        # a decode batch of 37 sequences through the 13B block's up projection
        dict(name="linear_batch", op="linear", T=37, K=5120, N=13824, y="bf16", bias=False, bits=6),
        # a 2,048-token prompt through the 70B block's up projection: matrix cores
        dict(name="linear_prompt", op="linear", T=2048, K=8192, N=28672, y="bf16", bias=False, bits=8),
        # one decode step of 8 sequences, 32 heads
        dict(name="append_decode", op="append", n_seq=8, max_q=1, max_len=2048, H=32, Hkv=32, d=128,
             page=64, x="bf16", s_a=True),
        # two prompts and ten decoding sequences in one batch, grouped heads
        dict(name="append_mixed", op="append", n_seq=12, max_q=4096, max_len=8192, H=64, Hkv=8, d=128,
             page=64, x="f32", s_a=False),
        # one sequence decoding at 2,048 tokens, 32 heads
        dict(name="attend_decode", op="attend", n_seq=1, max_q=1, max_len=2048, H=32, Hkv=32, d=128,
             page=64),
        # a serving batch of 64 sequences of ragged lengths, grouped heads
        dict(name="attend_batch", op="attend", n_seq=64, max_q=1, max_len=8192, H=64, Hkv=8, d=128,
             page=64),
        # one long conversation: a single row of queries over 131,072 tokens
        dict(name="attend_long", op="attend", n_seq=1, max_q=1, max_len=131072, H=64, Hkv=8, d=128,
             page=128),
        # prompt chunks of up to 2,048 tokens over a cached prefix
        dict(name="attend_prompt", op="attend", n_seq=2, max_q=2048, max_len=4096, H=32, Hkv=32, d=128,
             page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "append", "attend"])
    if op == "norm":
        D = 8 * _log(rng, 16, 1536)
        return dict(op=op, T=_log(rng, 1, max(1, min(16384, 100_000_000 // D))), D=D,
                    x=rng.choice(["bf16", "f32"]), r=rng.choice(["bf16", "f32", "none"]),
                    bias=rng.random() < 0.5, bits=rng.choice([4, 6, 8]))
    if op == "linear":
        K = 16 * _log(rng, 16, 1024)
        N = 8 * _log(rng, 16, 2048)
        return dict(op=op, T=_log(rng, 1, max(1, min(4096, 300_000_000_000 // (2 * K * N)))), K=K, N=N,
                    y=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.5, bits=rng.choice([4, 6, 8]))
    Hkv = rng.choice([1, 2, 4, 8, 16, 32])
    H = Hkv * rng.choice([g for g in (1, 2, 4, 5, 8) if Hkv * g <= 64])
    d = rng.choice([64, 128])
    page = rng.choice([32, 64, 128])
    c = dict(op=op, n_seq=_log(rng, 1, 64), H=H, Hkv=Hkv, d=d, page=page)
    if op == "append":
        budget = 16_000_000 // (c["n_seq"] * (H + 2 * Hkv) * d)       # new elements of a batch
        c["max_q"] = min(_log(rng, 1, 4096), max(1, budget))
        c["max_len"] = c["max_q"] + min(_log(rng, 64, 8192), max(64, 200_000_000 // (c["n_seq"] * Hkv * d)))
        return dict(c, x=rng.choice(["bf16", "f32"]), s_a=rng.random() < 0.5)
    # cached elements, then score elements, stay below the largest listed case's
    c["max_len"] = min(_log(rng, 64, 131072), max(64, 300_000_000 // (c["n_seq"] * Hkv * d)))
    q = max(1, 130_000_000 // (c["n_seq"] * c["max_len"] * H))
    c["max_q"] = min(_log(rng, 1, 2048), q, c["max_len"])
    return c


# ------------------------------------------------------------------ inputs
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _channels(g, n):
    """A width's channel scales: a few outlier channels, as language models' activations have."""
    s = torch.exp(0.3 * _normal(g, n))
    out = torch.rand(n, generator=g, device=DEV) < 0.005
    return torch.where(out, 20.0 * s, s)


def _plan(case):
    """Host lengths of a ragged batch: (tokens in the cache before the call, new tokens) per sequence.
    A sequence that gets more than one page of new tokens starts at a page's beginning; so a repeated
    append finds the rows it reads as they were."""
    n, P, mq, ml = case["n_seq"], case["page"], case["max_q"], case["max_len"]
    rng = random.Random(n * 1000003 + mq * 8191 + ml * 131 + P)
    mixed = case["op"] == "append" and n > 4             # decoding sequences beside two prompts
    new = [mq if i == 0 or mq == 1 else rng.randint(0, 3) if mixed and i >= 2 else rng.randint(1, mq)
           for i in range(n)]
    before = [ml - q if i == 0 else rng.randint(0 if q else 1, ml - q) for i, q in enumerate(new)]
    return [b - b % P if q > P else b for b, q in zip(before, new)], new


def _starts(counts):
    return list(itertools.accumulate(counts, initial=0))


def _to_k(x):
    """[..., P, d] -> the K pages' operand order [..., P * d]."""
    P, d = x.shape[-2:]
    lead = x.shape[:-2]
    n = len(lead)
    y = x.reshape(*lead, P // 16, 16, d // 64, 4, 16)
    return y.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*lead, P * d)


def _from_k(x, P, d):
    lead = x.shape[:-1]
    n = len(lead)
    y = x.reshape(*lead, P // 16, d // 64, 4, 16, 16)
    return y.permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).reshape(*lead, P, d)


def _to_v(x):
    """[..., P, d] -> the V pages' operand order [..., P * d]."""
    P, d = x.shape[-2:]
    lead = x.shape[:-2]
    n = len(lead)
    y = x.reshape(*lead, P // 32, 2, 4, 4, d // 32, 2, 16)          # c e1 g e0 jj hh r
    return y.permute(*range(n), n, n + 4, n + 2, n + 6, n + 5, n + 1, n + 3).reshape(*lead, P * d)


def _from_v(x, P, d):
    lead = x.shape[:-1]
    n = len(lead)
    y = x.reshape(*lead, P // 32, d // 32, 4, 16, 2, 2, 4)          # c jj g r hh e1 e0
    return y.permute(*range(n), n, n + 5, n + 2, n + 6, n + 1, n + 4, n + 3).reshape(*lead, P, d)


def _to_vw(x):
    """[..., P, d] -> the bf16 V windows' operand order [..., P * d]."""
    P, d = x.shape[-2:]
    lead = x.shape[:-2]
    n = len(lead)
    y = x.reshape(*lead, P // 32, 2, 4, 4, d // 16, 16)             # c e1 g e0 jt r
    return y.permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3).reshape(*lead, P * d)


def _from_vw(x, P, d):
    lead = x.shape[:-1]
    n = len(lead)
    y = x.reshape(*lead, P // 32, d // 16, 4, 16, 2, 4)             # c jt g r e1 e0
    return y.permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3).reshape(*lead, P, d)


def _quant_pages(x):
    """Symmetric 8-bit codes of [..., P, d] blocks, and their steps."""
    a = x.float().abs().amax((-2, -1))
    h = torch.clamp(a / 127.0, min=1e-5)
    q = torch.round(x.float() * (1.0 / h)[..., None, None])
    return torch.clamp(q, -127, 127), h


def _random_pages(g, m, Hkv, P, d, channels, order):
    """Codes (in operand order) and steps of m random pages, 256 pages' worth of memory at a time."""
    parts = [_quant_pages((_normal(g, min(256, m - j), Hkv, P, d) * channels).bfloat16())
             for j in range(0, m, 256)] or [_quant_pages(torch.zeros(0, Hkv, P, d, device=DEV))]
    return torch.cat([order(q.to(torch.int8)) for q, _ in parts]), torch.cat([h for _, h in parts])


def _cache(case, g, before, total):
    """A filled cache: pages in shuffled order, the open pages in the windows."""
    n, P, Hkv, d = case["n_seq"], case["page"], case["Hkv"], case["d"]
    need = [-(-t // P) for t in total]
    full = [b // P for b in before]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    # entries behind a sequence's last page are -1
    col = torch.arange(max(1, max(need)), device=DEV)
    at = torch.tensor(_starts(need)[:-1], device=DEV)[:, None] + col
    table = torch.where(col < torch.tensor(need, device=DEV)[:, None], perm[at.clamp(max=n_pages - 1)], -1)
    kc = 1.0 * _channels(g, Hkv * d).view(Hkv, 1, d)
    # full pages' codes and steps: rows' channel scales and a page's own level
    ids = table[col < torch.tensor(full, device=DEV)[:, None]].long()
    k_codes = torch.zeros(n_pages, Hkv, P * d, dtype=torch.int8, device=DEV)
    v_codes = torch.zeros_like(k_codes)
    k_scale = torch.zeros(n_pages, Hkv, device=DEV)
    v_scale = torch.zeros(n_pages, Hkv, device=DEV)
    k_codes[ids], k_scale[ids] = _random_pages(g, len(ids), Hkv, P, d, kc, _to_k)
    v_codes[ids], v_scale[ids] = _random_pages(g, len(ids), Hkv, P, d, torch.ones_like(kc), _to_v)
    k_win = (_normal(g, n, 2, Hkv, P, d) * kc).bfloat16()
    v_win = _normal(g, n, 2, Hkv, P, d).bfloat16()
    return dict(k_codes=k_codes, v_codes=v_codes, k_scale=k_scale, v_scale=v_scale,
                k_window=k_win.reshape(n, 2, Hkv, P * d), v_window=_to_vw(v_win), table=table)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "norm":
        T, D = case["T"], case["D"]
        ch = _channels(g, D)
        s["X"] = (_normal(g, T, D) * ch).to(_TYPE[case["x"]])
        s["R"] = None if case["r"] == "none" else (0.3 * _normal(g, T, D) * ch).to(_TYPE[case["r"]])
        s["gain"] = (1.0 + 0.2 * _normal(g, D)) / ch.sqrt()
        s["bias"] = 0.1 * _normal(g, D) if case["bias"] else None
        return s
    if case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        top = float(2 ** case["bits"] - 1)
        mid = top / 2 + 0.05 * top * _normal(g, T, 1)
        s["codes"] = torch.clamp(torch.round(mid + top / 7 * _normal(g, T, K)), 0, top).to(torch.uint8)
        s["h"] = 0.01 + 0.02 * torch.rand(T, generator=g, device=DEV)
        s["z"] = torch.round(mid.reshape(T))
        mid = top / 2 + 0.02 * top * _normal(g, N, 1)
        w = torch.clamp(torch.round(mid + top / 7 * _normal(g, N, K)), 0, top).to(torch.uint8)
        s["w"] = w
        s["h_w"] = 1e-3 * (0.5 + torch.rand(N, generator=g, device=DEV))
        s["z_w"] = torch.round(mid.reshape(N))
        s["B"] = _normal(g, N) if case["bias"] else None
        # the weight as a server keeps it: codes - 128 in operand order, and their sums
        Np, Kp = -(-N // 16) * 16, -(-K // 64) * 64
        b = torch.zeros(Np, Kp, dtype=torch.int8, device=DEV)
        b[:N, :K] = (w.to(torch.int16) - 128).to(torch.int8)
        s["wsum"] = (w.to(torch.int32) - 128).sum(1).to(torch.int32)
        s["packed"] = b.view(Np // 16, 16, Kp // 64, 4, 16).permute(0, 2, 3, 1, 4).contiguous()
        return s
    n, H, Hkv, d, P = case["n_seq"], case["H"], case["Hkv"], case["d"], case["page"]
    before, new = _plan(case)
    total = [b + q for b, q in zip(before, new)]
    start = _starts(new)
    T = start[-1]
    # attention reads a cache that holds the new tokens already
    s.update(_cache(case, g, total if case["op"] == "attend" else before, total))
    s["length"], s["q_start"], s["T"] = _ints(before), _ints(start), T
    s["max_q"] = max(new)
    s["seq"] = torch.repeat_interleave(torch.arange(n, device=DEV), _ints(new).long())
    s["pos"] = torch.arange(T, device=DEV) - s["q_start"].long()[s["seq"]] + s["length"].long()[s["seq"]]
    if case["op"] == "attend":
        s["Q"] = _normal(g, T, H * d).bfloat16()
        return s
    # one row of q, k and v per token, as the stacked projection leaves it
    s["qkv"] = _normal(g, T, (H + 2 * Hkv) * d).to(_TYPE[case["x"]])
    s["s_a"] = (0.5 + torch.rand(Hkv * d, generator=g, device=DEV)) if case["s_a"] else None
    ang = (torch.arange(max(total), device=DEV, dtype=torch.float64)[:, None]
           * 10000.0 ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d))
    s["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float()
    # the rows of every page that the call touches
    first = [b - b % P for b in before]
    rows = [t - f for t, f in zip(total, first)]
    rstart = _starts(rows)
    s["first"], s["row_start"], s["rows"], s["max_rows"] = _ints(first), _ints(rstart), rstart[-1], max(rows)
    s["rseq"] = torch.repeat_interleave(torch.arange(n, device=DEV), _ints(rows).long())
    s["rpos"] = (torch.arange(rstart[-1], device=DEV) - s["row_start"].long()[s["rseq"]]
                 + s["first"].long()[s["rseq"]])
    return s


# ------------------------------------------------------------------ one pass
def _values(codes, h, z):
    """The values that integer codes stand for."""
    return ((codes.float() - z[:, None]) * h[:, None]).bfloat16()


def _own_cache(s):
    from paper_2308_13137_amd import oq
    c = s["case"]
    return oq.KVCache.of(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_window"],
                         s["v_window"], page=c["page"], head_dim=c["d"])


def run(s):
    op = s["case"]["op"]
    return {"norm": _norm, "linear": _linear, "append": _append, "attend": _attend}[op](s)


def _norm(s):
    case, X, R = s["case"], s["X"], s["R"]
    if own:
        from paper_2308_13137_amd import oq
        H, values, _, h, _ = oq.rmsnorm_quant(X, s["gain"], case["bits"], R=R, bias=s["bias"], eps=1e-6,
                                              dq_dtype=torch.bfloat16)
        return dict(H=H, values=values, h=h)
    H = X if R is None else (X.float() + R.float()).to(X.dtype)
    f = H.float()
    y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + 1e-6) * s["gain"]
    if s["bias"] is not None:
        y = y + s["bias"]
    top = float(2 ** case["bits"] - 1)
    hi, lo = y.amax(1), y.amin(1)
    h = torch.clamp((hi - lo) / top, min=1e-5)
    z = -torch.round(lo / h)
    q = torch.clamp(torch.round(y / h[:, None]) + z[:, None], 0, top)
    return dict(H=H, values=_values(q, h, z), h=h)


def _linear(s):
    case = s["case"]
    if own:
        from paper_2308_13137_amd import oq
        return oq.int8_linear(s["codes"], s["h"], s["z"], s["packed"], s["wsum"], s["h_w"], s["z_w"],
                              B=s["B"], out_dtype=_TYPE[case["y"]])
    a = s["codes"].float() - s["z"][:, None]
    b = s["w"].float() - s["z_w"][:, None]
    y = (a @ b.t()) * s["h"][:, None] * s["h_w"]
    if s["B"] is not None:
        y = y + s["B"]
    return y.to(_TYPE[case["y"]])


def _append(s):
    case = s["case"]
    n, H, Hkv, d, P = case["n_seq"], case["H"], case["Hkv"], case["d"], case["page"]
    qkv, T = s["qkv"], s["T"]
    Q, K, V = qkv[:, :H * d], qkv[:, H * d:(H + Hkv) * d], qkv[:, (H + Hkv) * d:]
    if own:
        cache = _own_cache(s)
        q = cache.append(Q, K, V, s["table"], s["length"], s["q_start"], s["max_q"], rope=s["rope"],
                         s_a=s["s_a"])
        k, v = cache.read(s["table"], s["first"], s["length"], s["q_start"], s["row_start"], s["rows"],
                          s["max_rows"])
        return dict(Q=q, K=k, V=v)
    cs, sn = s["rope"][s["pos"], :, 0][:, None], s["rope"][s["pos"], :, 1][:, None]
    sa = s["s_a"].view(Hkv, d) if s["s_a"] is not None else torch.ones(Hkv, d, device=DEV)

    def turn(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)

    q = (turn(Q.reshape(T, H, d).float()) / sa.repeat_interleave(H // Hkv, 0)).bfloat16().view(T, H * d)
    k = (turn(K.reshape(T, Hkv, d).float()) * sa).bfloat16()
    v = V.reshape(T, Hkv, d).bfloat16()
    # the touched pages of every sequence, padded to the longest: old rows from the windows, then new
    m = -(-s["max_rows"] // P) * P
    first, ln = s["first"].long(), s["length"].long()
    half = (first // P) % 2
    i = torch.arange(n, device=DEV)
    total = ln + (s["q_start"][1:] - s["q_start"][:-1]).long()
    full = (first[:, None] + P * (1 + torch.arange(m // P, device=DEV))) <= total[:, None]

    def cached(x, win):
        rows = torch.zeros(n, m, Hkv, d, dtype=torch.bfloat16, device=DEV)
        rows[:, :P] = win[i, half].transpose(1, 2)
        rows[torch.arange(m, device=DEV) >= (ln - first)[:, None]] = 0
        rows[s["seq"], s["pos"] - first[s["seq"]]] = x
        blocks = rows.view(n, m // P, P, Hkv, d).transpose(2, 3)
        code, h = _quant_pages(blocks)
        deq = (code * h[..., None, None]).bfloat16()
        rows = torch.where(full[:, :, None, None, None], deq, blocks).transpose(2, 3).reshape(n, m, Hkv * d)
        return rows[s["rseq"], s["rpos"] - first[s["rseq"]]]

    return dict(Q=q, K=cached(k, s["k_window"].view(n, 2, Hkv, P, d)),
                V=cached(v, _from_vw(s["v_window"], P, d)))


def _dequantised(s, kind):
    """[n_seq, max tokens, Hkv, d] fp32 of the cached rows (rows behind a sequence's end are anything finite)."""
    case = s["case"]
    n, Hkv, d, P = case["n_seq"], case["Hkv"], case["d"], case["page"]
    total = s["length"].long() + (s["q_start"][1:] - s["q_start"][:-1]).long()
    pages = s["table"].long().clamp(min=0)
    codes, scale = (s["k_codes"], s["k_scale"]) if kind == "k" else (s["v_codes"], s["v_scale"])
    x = codes[pages]
    x = (_from_k(x, P, d) if kind == "k" else _from_v(x, P, d)).float() * scale[pages][..., None, None]
    win = s["k_window"].view(n, 2, Hkv, P, d) if kind == "k" else _from_vw(s["v_window"], P, d)
    i = torch.arange(n, device=DEV)
    open_page = (total // P).clamp(max=pages.shape[1] - 1)
    part = (total % P != 0)[:, None, None, None]
    x[i, open_page] = torch.where(part, win[i, open_page % 2].float(), x[i, open_page])
    return x.transpose(2, 3).reshape(n, -1, Hkv, d)


def _attend(s):
    case = s["case"]
    n, H, Hkv, d = case["n_seq"], case["H"], case["Hkv"], case["d"]
    if own:
        return _own_cache(s).attend(s["Q"], s["table"], s["length"], s["q_start"], s["max_q"])
    G, T, mq = H // Hkv, s["T"], s["max_q"]
    k, v = _dequantised(s, "k"), _dequantised(s, "v")
    q = torch.zeros(n, mq, Hkv, G, d, device=DEV)
    j = torch.arange(T, device=DEV) - s["q_start"].long()[s["seq"]]
    q[s["seq"], j] = s["Q"].view(T, Hkv, G, d).float()
    q = q.permute(0, 2, 1, 3, 4).reshape(n * Hkv, mq * G, d)
    k = k.permute(0, 2, 1, 3).reshape(n * Hkv, -1, d)
    v = v.permute(0, 2, 1, 3).reshape(n * Hkv, -1, d)
    sc = torch.bmm(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
    last = s["length"].long()[:, None] + torch.arange(mq, device=DEV)
    hide = torch.arange(k.shape[1], device=DEV) > last[..., None]
    sc = sc.view(n, Hkv, mq, G, -1).masked_fill_(hide[:, None, :, None], -math.inf)
    sc = torch.exp(sc - sc.amax(-1, keepdim=True))
    sc = sc / sc.sum(-1, keepdim=True)
    o = torch.bmm(sc.view(n * Hkv, mq * G, -1), v).view(n, Hkv, mq, G, d).permute(0, 2, 1, 3, 4)
    return o[s["seq"], j].reshape(T, H * d).bfloat16()


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = {"bf16": 2, "f32": 4, "none": 0}
    if case["op"] == "norm":
        n = case["T"] * case["D"]
        x, r = size[case["x"]], size[case["r"]]
        return dict(bytes=n * (x + r + (x if r else 0) + 1) + 4 * case["D"] * (1 + case["bias"])
                    + 8 * case["T"], flops=8 * n)
    if case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        return dict(bytes=T * K + N * K + T * N * size[case["y"]] + 8 * T + 12 * N, flops=2 * T * K * N)
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    before, new = _plan(case)
    T, total = sum(new), sum(before) + sum(new)
    if case["op"] == "append":
        # the new rows in, the turned queries out, codes or bf16 rows into the cache and out again
        return dict(bytes=T * d * ((H + 2 * Hkv) * size[case["x"]] + 2 * H + 2 * Hkv * (1 + 1 + 2))
                    + 4 * T * d, flops=6 * T * d * (H + Hkv))
    pairs = sum(q * b + q * (q + 1) // 2 for b, q in zip(before, new))
    return dict(bytes=2 * total * Hkv * d + 4 * T * H * d, flops=4 * H * d * pairs)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        H = s["X"].double()
        if s["R"] is not None:
            H = (H + s["R"].double()).to(s["X"].dtype).double()
        y = H / (H.square().sum(1, keepdim=True) / H.shape[1] + 1e-6).sqrt() * s["gain"].double()
        y = y + (0 if s["bias"] is None else s["bias"].double())
        n = 2 ** case["bits"] - 1
        lo = y.min(1).values
        h = ((y.max(1).values - lo) / n).clamp_min(1e-5)
        z = -(lo / h).round()
        q = ((y / h[:, None]).round() + z[:, None]).clamp(0, n)
        return dict(H=H, values=(q - z[:, None]) * h[:, None], h=h)
    if case["op"] == "linear":
        a = (s["codes"].double() - s["z"].double()[:, None]) * s["h"].double()[:, None]
        w = s["w"]
        out = torch.empty(case["T"], case["N"], dtype=torch.float64, device=DEV)
        for j in range(0, case["N"], 4096):
            b = w[j:j + 4096].double() - s["z_w"][j:j + 4096].double()[:, None]
            out[:, j:j + 4096] = a @ (b * s["h_w"][j:j + 4096].double()[:, None]).t()
        return out if s["B"] is None else out + s["B"].double()
    n, H, Hkv, d, P = case["n_seq"], case["H"], case["Hkv"], case["d"], case["page"]
    length, start = s["length"].tolist(), s["q_start"].tolist()
    G = H // Hkv
    if case["op"] == "append":
        c, si = s["rope"][s["pos"]].double().unbind(-1)
        z = torch.complex(c, si)[:, None]
        x = s["qkv"].double().view(s["T"], H + 2 * Hkv, d)
        t = x[:, :H + Hkv]
        t = torch.complex(t[..., :d // 2], t[..., d // 2:]) * z
        t = torch.cat([t.real, t.imag], -1)
        if s["s_a"] is not None:
            sa = s["s_a"].double().view(Hkv, 1, d)
            t = torch.cat([(t[:, :H].reshape(-1, Hkv, G, d) / sa).reshape(-1, H, d), t[:, H:] * sa[:, 0]], 1)
        ks, vs = [], []
        kw, vw = s["k_window"].view(n, 2, Hkv, P, d), _from_vw(s["v_window"], P, d)
        for i in range(n):
            f, L, b, e = length[i] - length[i] % P, length[i], start[i], start[i + 1]
            half = (f // P) % 2
            for w, new, out in ((kw, t[b:e, H:], ks), (vw, x[b:e, H + Hkv:], vs)):
                r = torch.cat([w[i, half, :, :L - f].transpose(0, 1).double(), new.bfloat16().double()])
                m = len(r) // P * P
                blk = r[:m].view(-1, P, Hkv, d)
                h = (blk.abs().amax((1, 3), keepdim=True) / 127).clamp_min(1e-5)
                out.append(torch.cat([((blk / h).round().clamp(-127, 127) * h).view(m, Hkv, d), r[m:]])
                           .reshape(-1, Hkv * d))
        return dict(Q=t[:, :H].reshape(-1, H * d), K=torch.cat(ks), V=torch.cat(vs))
    out = torch.empty(s["T"], H, d, dtype=torch.float64, device=DEV)
    kw, vw = s["k_window"].view(n, 2, Hkv, P, d), _from_vw(s["v_window"], P, d)
    for i in range(n):
        b, e = start[i], start[i + 1]
        tot, m = length[i] + e - b, (length[i] + e - b) // P
        pages = s["table"][i, :m].long()
        for u in range(Hkv):
            k = _from_k(s["k_codes"][pages, u], P, d).double() * s["k_scale"][pages, u].double()[:, None, None]
            v = _from_v(s["v_codes"][pages, u], P, d).double() * s["v_scale"][pages, u].double()[:, None, None]
            k = torch.cat([k.reshape(-1, d), kw[i, m % 2, u, :tot - m * P].double()])
            v = torch.cat([v.reshape(-1, d), vw[i, m % 2, u, :tot - m * P].double()])
            for h in range(u * G, u * G + G):
                w = s["Q"][b:e, h * d:h * d + d].double() @ k.t() / math.sqrt(d)
                w = w + torch.full_like(w, -math.inf).triu(length[i] + 1)
                out[b:e, h] = w.softmax(1) @ v
    return out.view(s["T"], H * d)
