"""The operators that stand between the attention and the Linear layers of a video DiT block, as a
user's program calls them.

Three families, all through the public binding (`paper_2512_16093_amd.binding`):

  rope    rotary positions over the token grid's axes (time, height, width) on q and k, with the
          root-mean-square norm of the queries and keys on the way: what a QKV projection leaves
          becomes what `sla_attention_fwd` takes.  "fwd": `rope_qk_fwd`; "bwd": `rope_qk_bwd`.
  norm    root-mean-square norm with the addition to the residual stream.  "linear": its result
          goes, as 8-bit codes with block scales, into a W8A8 Linear layer (`w8a8_norm_linear_fwd`);
          "fwd": bf16 (`norm_rms_fwd`); "bwd": `norm_rms_bwd`.
  cross   attention to an encoder's states of another length, padded prompts of a batch included.
          "fwd": `xattn_fwd`; "train": `xattn_fwd` with the log-sum-exp, then `xattn_bwd`.

Where `own` is false the same functions are computed in their plain form, in 32 bits (the angles of
the positions in 64) and rounded once at the end.  The residual stream h = x + res is a bf16 tensor of the
operator's definition, and the norm is that of the stored stream: what a backward pass, which finds the
stored one, differentiates.
"""
import math

import torch

own = False

D = 128
AXES = (22, 21, 21)      # channel pairs of (time, height, width): 44, 42 and 42 of 128 channels
THETA = 10000.0
EPS = 1e-6


def _rope(pass_, grid, heads, norm, batch=1, packed=False, pairing="interleaved", start=0):
    return {"family": "rope", "pass": pass_, "batch": batch, "heads": heads, "grid_t": grid[0], "grid_h": grid[1],
            "grid_w": grid[2], "start": start, "norm": norm, "packed": packed, "pairing": pairing}


def _norm(pass_, tokens, features, outputs=0, residual=True, bias=False):
    return {"family": "norm", "pass": pass_, "tokens": tokens, "features": features, "outputs": outputs,
            "residual": residual, "bias": bias}


def _cross(pass_, queries, keys, heads, kv_heads=None, batch=1, short=1.0, token_major=True):
    return {"family": "cross", "pass": pass_, "batch": batch, "queries": queries, "keys": keys, "heads": heads,
            "kv_heads": kv_heads or heads, "short": short, "token_major": token_major}


def listed():
    cases = {
        # the repository's tiny grid: a latency measurement
        "rope_tiny": _rope("fwd", (4, 16, 16), 2, "none"),
        # the large 720P model: q and k out of the packed projection, normed over all heads, head-major for the attention
        "rope_720p_h40": _rope("fwd", (21, 45, 80), 40, "token", packed=True),
        # finetuning the small 480P model: the gradients back through rotation and norm, the norms' weights included
        "rope_480p_h12_bwd": _rope("bwd", (21, 30, 52), 12, "token"),
        # a step on one token (a conditioning vector of the large model): latency and the weight's bytes
        "norm_linear_one_token": _norm("linear", 1, 5120, 5120, bias=True),
        # the small 480P model's stream, normed and quantised into the feed-forward's first product
        "norm_linear_480p_up": _norm("linear", 32760, 1536, 8960, bias=True),
        # the large 720P model's stream into an attention projection
        "norm_linear_720p_proj": _norm("linear", 75600, 5120, 5120, bias=True),
        # training: the norm in bf16 at the small model's width, and its gradient at the large one's
        "norm_480p_fwd": _norm("fwd", 32760, 1536),
        "norm_720p_bwd": _norm("bwd", 75600, 5120),
        # one query token against a long memory, four query heads to a key head
        "cross_one_token_long": _cross("fwd", 1, 32760, 40, kv_heads=10),
        # a guided pair of samples in one batch: a full prompt, and a short one padded to the same length
        "cross_480p_pair": _cross("fwd", 32760, 512, 12, batch=2, short=0.25),
        # the large 720P model's cross attention to a prompt of 512 states
        "cross_720p_h40": _cross("fwd", 75600, 512, 40),
        # finetuning the small 480P model: forward and backward
        "cross_480p_train": _cross("train", 32760, 512, 12, short=1.0),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _limit():
    return max(work(c)["flops"] for c in listed())


def draw(rng):
    """One more call of the same ranges: 1 to 75 600 tokens, 1 to 40 heads, every norm and pairing; widths of
    8 to 13 824; prompts of 1 to 8192 states, whole, short or empty, with key heads shared or not."""
    family = rng.choice(("rope", "norm", "cross"))
    if family == "rope":
        N = _log_int(rng, 1, 75600)
        t = rng.randint(1, 21)
        h = max(1, int(round(math.sqrt(N / t) * rng.uniform(0.6, 1.0))))
        w = max(1, int(N / (t * h)))
        case = _rope(rng.choice(("fwd", "fwd", "bwd")), (t, h, w), _log_int(rng, 1, 40), rng.choice(("none", "head", "token")),
                     batch=rng.choice((1, 1, 2)), packed=rng.random() < 0.5,
                     pairing=rng.choice(("interleaved", "interleaved", "halves")), start=rng.choice((0, rng.randint(1, 100000))))
        while _tokens(case) * case["batch"] * case["heads"] > 75600 * 40:
            case["batch"], case["heads"] = 1, max(1, case["heads"] * 2 // 3)
        return case
    if family == "norm":
        pass_ = rng.choice(("linear", "linear", "fwd", "bwd"))
        tokens = _log_int(rng, 1, 75600)
        if pass_ == "linear":
            case = _norm(pass_, tokens, 128 * _log_int(rng, 1, 108), 128 * _log_int(rng, 1, 108), residual=rng.random() < 0.7,
                         bias=rng.random() < 0.7)
        else:
            case = _norm(pass_, tokens, 8 * _log_int(rng, 1, 1728), residual=rng.random() < 0.7)
        while work(case)["flops"] > _limit() or case["tokens"] * case["features"] > 75600 * 5120:
            case["tokens"] = max(1, case["tokens"] * 2 // 3)
        return case
    kv_heads = _log_int(rng, 1, 40)
    batch = rng.choice((1, 1, 2, 3))
    case = _cross(rng.choice(("fwd", "fwd", "train")), _log_int(rng, 1, 75600), _log_int(rng, 1, 8192),
                  kv_heads * rng.choice([g for g in (1, 1, 2, 4, 5) if g * kv_heads <= 40]), kv_heads=kv_heads, batch=batch,
                  short=rng.choice((1.0, round(rng.uniform(0.05, 1.0), 3)) if batch == 1 else (1.0, round(rng.random(), 3), 0.0)),
                  token_major=rng.random() < 0.6)
    # the score matrix of the largest listed case, and half of it where three matrices of that kind are kept
    most = 75600 * 512 * 40 // (2 if case["pass"] == "train" else 1)
    while case["batch"] * case["heads"] * case["queries"] * case["keys"] > most:
        case["batch"], case["queries"] = 1, max(1, case["queries"] * 2 // 3)
    return case


def _tokens(case):
    return case["grid_t"] * case["grid_h"] * case["grid_w"]


def _lens(case):
    """Keys of each sample: every second prompt is the short one."""
    short = int(case["keys"] * case["short"])
    return [max(1, short)] if case["batch"] == 1 else [case["keys"] if i % 2 == 0 else short for i in range(case["batch"])]


def work(case):
    if case["family"] == "rope":
        elems = 2 * case["batch"] * _tokens(case) * case["heads"] * D          # of q and k
        tensors = 2 if case["pass"] == "fwd" else 3 if case["norm"] != "none" else 2
        return {"bytes": 2 * elems * tensors + 12 * _tokens(case), "flops": elems * (3 if case["norm"] == "none" else 7)}
    if case["family"] == "norm":
        M, K, N = case["tokens"], case["features"], case["outputs"]
        res = case["residual"]
        if case["pass"] == "linear":
            # x (and res, h), the weight's codes, y; the codes of the activations stay within the call
            return {"bytes": 2 * M * K * (3 if res else 1) + N * K + 2 * M * N, "flops": 2 * M * N * K + 5 * M * K}
        if case["pass"] == "fwd":
            return {"bytes": 2 * M * K * (4 if res else 2), "flops": 5 * M * K}
        return {"bytes": 2 * M * K * (4 if res else 3) + 4 * K, "flops": 12 * M * K}
    pairs = case["heads"] * case["queries"] * sum(_lens(case))
    rows = case["batch"] * case["queries"] * case["heads"] * D
    kv = sum(_lens(case)) * case["kv_heads"] * D
    if case["pass"] == "fwd":
        return {"bytes": 2 * (2 * rows + 2 * kv), "flops": 4 * pairs * D}
    # q, k, v, dO in; O, dq, dk, dv out
    return {"bytes": 2 * (4 * rows + 4 * kv), "flops": 14 * pairs * D}


# ---------------------------------------------------------------------------
# What a program has in hand before the call.
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _bf16(shape, gen, amp=1.0):
    """Normal values in bf16, a slab at a time (the largest tensor in 32 bits would be as large as everything else)."""
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = x.view(-1)
    for part in flat.split(1 << 27):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(amp))
    return x


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": case}
    if own:
        from paper_2512_16093_amd import binding
        s["b"] = binding
    if case["family"] == "rope":
        B, H, N = case["batch"], case["heads"], _tokens(case)
        # the token grid's coordinates, row by row, behind `start` frames that a longer video has had before
        n = torch.arange(N, device="cuda")
        hw = case["grid_h"] * case["grid_w"]
        s["pos"] = torch.stack((n // hw + case["start"], n // case["grid_w"] % case["grid_h"], n % case["grid_w"]), 1).int().contiguous()

        def pair(amp):
            if case["packed"]:      # the projection's [B, N, 3, H, d]
                x = _bf16((B, N, 3, H, D), gen, amp)
                return x[:, :, 0].permute(0, 2, 1, 3), x[:, :, 1].permute(0, 2, 1, 3)
            return [_bf16((B, N, H, D), gen, amp).permute(0, 2, 1, 3) for _ in range(2)]

        s["q"], s["k"] = pair(1.7)
        if case["pass"] == "bwd":
            s["dq_out"], s["dk_out"] = pair(0.01)
        width = {"none": 0, "head": D, "token": H * D}[case["norm"]]
        s["qw"], s["kw"] = [(1 + 0.2 * torch.randn(width, generator=gen, device="cuda")).bfloat16() if width else None for _ in range(2)]
        if own:
            s["plan"] = s["b"].rope_make_plan(AXES, THETA, case["pairing"])
        return s
    if case["family"] == "norm":
        M, K, N = case["tokens"], case["features"], case["outputs"]
        # a residual stream: a few features much larger than the others, a token's amplitude its own
        x = _bf16((M, K), gen)
        outlier = torch.randperm(K, generator=gen, device="cuda")[:max(1, K // 100)]
        x[:, outlier] *= (10.0 + 20.0 * torch.rand((outlier.numel(),), generator=gen, device="cuda")).bfloat16()
        x *= (0.5 + 1.5 * torch.rand((M, 1), generator=gen, device="cuda")).bfloat16()
        s["x"] = x
        s["res"] = _bf16((M, K), gen, 0.01 if case["pass"] == "bwd" else 0.3) if case["residual"] else None
        s["w"] = (1 + 0.2 * torch.randn(K, generator=gen, device="cuda")).bfloat16()
        if case["pass"] == "bwd":
            s["dy"] = _bf16((M, K), gen, 0.01)     # (and `res` is the gradient that comes down the residual stream)
        if case["pass"] == "linear":
            weight = (torch.randn((N, K), generator=gen, device="cuda") / math.sqrt(K)).bfloat16()
            s["bias"] = (0.1 * torch.randn(N, generator=gen, device="cuda")).bfloat16() if case["bias"] else None
            # the weight, quantised once: as the values its codes stand for, and as the framework's weight object
            s["weight"] = _blocks_8bit(weight.double()).float()
            if own:
                s["wq"] = s["b"].w8a8_quantize_weight(weight)
        return s
    B, H, G, Nq, Nk = case["batch"], case["heads"], case["kv_heads"], case["queries"], case["keys"]

    def heads(n, h, amp):
        if case["token_major"]:
            return _bf16((B, n, h, D), gen, amp).permute(0, 2, 1, 3)
        return _bf16((B, h, n, D), gen, amp)

    # normed queries and keys under weights that make a prompt's states differ; values as a projection leaves them
    s["q"], s["k"], s["v"] = heads(Nq, H, 1.5), heads(Nk, G, 1.5), heads(Nk, G, 1.0)
    lens = _lens(case)
    s["lens"] = None if min(lens) == Nk else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["pass"] == "train":
        s["dout"] = heads(Nq, H, 0.01)
    return s


# ---------------------------------------------------------------------------
# Plain forms.
# ---------------------------------------------------------------------------
def _angles(pos, dtype):
    """cos and sin [N, 64] of every channel pair's angle: pair j of an axis of n turns by theta^(-j / n) a step."""
    parts = []
    for a, n in enumerate(AXES):
        freq = THETA ** (-torch.arange(n, dtype=torch.float64, device=pos.device) / n)
        parts.append(pos[:, a:a + 1].double() * freq)
    ang = torch.cat(parts, 1)
    return ang.cos().to(dtype), ang.sin().to(dtype)


def _split(x, pairing):
    return (x[..., 0::2], x[..., 1::2]) if pairing == "interleaved" else (x[..., :D // 2], x[..., D // 2:])


def _join(a, b, pairing):
    return torch.stack((a, b), -1).flatten(-2) if pairing == "interleaved" else torch.cat((a, b), -1)


def _rotate(x, cos, sin, pairing):
    a, b = _split(x, pairing)
    return _join(a * cos - b * sin, a * sin + b * cos, pairing)


def _norm_dims(norm):
    return (1, 3) if norm == "token" else (3,)     # of a [B, H, N, d] tensor


def _norm_weight(w, norm, H):
    return w.view(1, H, 1, D) if norm == "token" else w.view(1, 1, 1, D)


def _rope_fwd_plain(x, w, cos, sin, case):
    x = x.to(cos.dtype)
    if case["norm"] != "none":
        x = x * torch.rsqrt((x * x).mean(_norm_dims(case["norm"]), keepdim=True) + EPS)
        x = x * _norm_weight(w.to(x.dtype), case["norm"], case["heads"])
    return _rotate(x, cos, sin, case["pairing"])


def _rope_bwd_plain(dy, x, w, cos, sin, case):
    """The gradient of x, and of the norm's weight (None without a norm)."""
    g = _rotate(dy.to(cos.dtype), cos, -sin, case["pairing"])
    if case["norm"] == "none":
        return g, None
    x, dims = x.to(cos.dtype), _norm_dims(case["norm"])
    r = torch.rsqrt((x * x).mean(dims, keepdim=True) + EPS)
    xhat = x * r
    dw = g * xhat
    dw = dw.sum((0, 2)).flatten() if case["norm"] == "token" else dw.sum((0, 1, 2))
    g = g * _norm_weight(w.to(x.dtype), case["norm"], case["heads"])
    return r * (g - xhat * (g * xhat).mean(dims, keepdim=True)), dw


def _blocks_8bit(y):
    """The values that the 8-bit codes of y's blocks of 128 x 128 stand for: scale max|block| / 127, nearest code, ties to even."""
    M, K = y.shape
    rows = -(-M // 128) * 128
    p = torch.cat((y, y.new_zeros((rows - M, K)))) if rows > M else y
    p = p.view(rows // 128, 128, K // 128, 128)
    amax = p.abs().amax((1, 3), keepdim=True)
    amax = torch.where(amax > 0, amax, torch.full_like(amax, 127.0))
    return (torch.round(p * 127.0 / amax) * (amax / 127.0)).view(rows, K)[:M]


def _norm_fwd_plain(x, res, w, dtype):
    """(h, y): the stream as it is stored, and its norm."""
    h = x if res is None else (x.to(dtype) + res.to(dtype)).bfloat16()
    v = h.to(dtype)
    return h, v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * w.to(dtype)


def _norm_bwd_plain(dy, dh, h, w, dtype):
    v, dy = h.to(dtype), dy.to(dtype)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    vhat = v * r
    g = dy * w.to(dtype)
    dx = r * (g - vhat * (g * vhat).mean(1, keepdim=True))
    return (dx if dh is None else dx + dh.to(dtype)), (dy * vhat).sum(0)


def _weights(q, k, lens):
    """exp(s - max) over each query's keys [B, G, rows, Nk] (zero where there are none), their sums, for q [B, G, rows, d]."""
    s = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    if lens is not None:
        s.masked_fill_(torch.arange(k.shape[2], device=q.device) >= lens.view(-1, 1, 1, 1), -math.inf)
    m = s.amax(3, keepdim=True)
    p = s.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    l = p.sum(3, keepdim=True)
    return p, torch.where(l > 0, 1.0 / l, torch.zeros_like(l))


def _grouped(x, G, dtype):
    """[B, H, n, d] with the query heads of a key head side by side: [B, G, H / G * n, d]."""
    B, H, n, _ = x.shape
    return x.to(dtype).contiguous().view(B, G, H // G * n, D)


def _cross_fwd_plain(s, dtype):
    q, k, v = _grouped(s["q"], s["k"].shape[1], dtype), s["k"].to(dtype).contiguous(), s["v"].to(dtype).contiguous()
    if s["lens"] is not None:
        v = v * (torch.arange(k.shape[2], device=q.device).view(1, 1, -1, 1) < s["lens"].view(-1, 1, 1, 1))
    p, inv = _weights(q, k, s["lens"])
    return (torch.matmul(p, v) * inv).view(s["q"].shape)


def _cross_train_plain(s, dtype):
    G = s["k"].shape[1]
    q, k, v = _grouped(s["q"], G, dtype), s["k"].to(dtype).contiguous(), s["v"].to(dtype).contiguous()
    do = _grouped(s["dout"], G, dtype)
    p, inv = _weights(q, k, s["lens"])
    p *= inv
    out = torch.matmul(p, v)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * out).sum(3, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(D))
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    return out.view(s["q"].shape), dq.view(s["q"].shape), dk, dv


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------
def _run_own(s):
    case, b = s["case"], s["b"]
    if case["family"] == "rope":
        if case["pass"] == "fwd":
            q, k = b.rope_qk_fwd(s["q"], s["k"], s["pos"], s["plan"], q_weight=s["qw"], k_weight=s["kw"], norm=case["norm"], eps=EPS)
            return {"q": q, "k": k}
        dq, dk, dqw, dkw = b.rope_qk_bwd(s["dq_out"], s["dk_out"], s["pos"], s["plan"], q=s["q"], k=s["k"], q_weight=s["qw"],
                                         k_weight=s["kw"], norm=case["norm"], eps=EPS)
        return {"dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw}
    if case["family"] == "norm":
        if case["pass"] == "linear":
            y, h = b.w8a8_norm_linear_fwd(s["x"], s["w"], s["wq"], case["outputs"], res=s["res"], eps=EPS, bias=s["bias"])
            return {"y": y, "h": h}
        if case["pass"] == "fwd":
            y, h = b.norm_rms_fwd(s["x"], s["w"], res=s["res"], eps=EPS)
            return {"y": y, "h": h}
        dx, dw = b.norm_rms_bwd(s["dy"], s["x"], s["w"], dh=s["res"], eps=EPS)
        return {"dx": dx, "dw": dw}
    if case["pass"] == "fwd":
        return {"out": b.xattn_fwd(s["q"], s["k"], s["v"], k_lens=s["lens"])[0]}
    out, lse = b.xattn_fwd(s["q"], s["k"], s["v"], k_lens=s["lens"], want_lse=True)
    dq, dk, dv = b.xattn_bwd(s["q"], s["k"], s["v"], out, s["dout"], lse, k_lens=s["lens"])
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    if case["family"] == "rope":
        cos, sin = _angles(s["pos"], torch.float32)
        if case["pass"] == "fwd":
            return {"q": _rope_fwd_plain(s["q"], s["qw"], cos, sin, case).bfloat16(),
                    "k": _rope_fwd_plain(s["k"], s["kw"], cos, sin, case).bfloat16()}
        dq, dqw = _rope_bwd_plain(s["dq_out"], s["q"], s["qw"], cos, sin, case)
        dk, dkw = _rope_bwd_plain(s["dk_out"], s["k"], s["kw"], cos, sin, case)
        return {"dq": dq.bfloat16(), "dk": dk.bfloat16(), "dqw": dqw, "dkw": dkw}
    if case["family"] == "norm":
        if case["pass"] == "bwd":
            dx, dw = _norm_bwd_plain(s["dy"], s["res"], s["x"], s["w"], torch.float32)
            return {"dx": dx.bfloat16(), "dw": dw}
        h, y = _norm_fwd_plain(s["x"], s["res"], s["w"], torch.float32)
        if case["pass"] == "linear":
            y = torch.matmul(_blocks_8bit(y), s["weight"].t())
            y = y if s["bias"] is None else y + s["bias"].float()
        return {"y": y.bfloat16(), "h": h}
    if case["pass"] == "fwd":
        return {"out": _cross_fwd_plain(s, torch.float32).bfloat16()}
    return dict(zip(("out", "dq", "dk", "dv"), (x.bfloat16() for x in _cross_train_plain(s, torch.float32))))


# ---------------------------------------------------------------------------
# The definitions in 64 bits, written apart from the plain forms.
# ---------------------------------------------------------------------------
def _exact_rope(case, s):
    B, H, N = case["batch"], case["heads"], _tokens(case)
    idx = torch.arange(D // 2, device="cuda")
    if case["pairing"] == "interleaved":
        lo, hi = 2 * idx, 2 * idx + 1
    else:
        lo, hi = idx, idx + D // 2
    # the rotation as a complex factor e^(i angle) of the number lo + i hi
    turn = torch.empty((N, D // 2), dtype=torch.float64, device="cuda")
    at = 0
    for axis, count in enumerate(AXES):
        for j in range(count):
            turn[:, at + j] = s["pos"][:, axis].double() / THETA ** (j / count)
        at += count
    factor = torch.polar(torch.ones_like(turn), turn)

    def one(x, w, dy):
        out = torch.empty((B, H, N, D), dtype=torch.float64, device="cuda")
        dw = torch.zeros((H, D), dtype=torch.float64, device="cuda")
        for i in range(B):
            x64 = x[i].double()
            if case["norm"] == "token":
                scale = (x64.pow(2).sum((0, 2)) / (H * D) + EPS).pow(-0.5).view(1, N, 1)
                gain = w.double().view(H, 1, D)
            elif case["norm"] == "head":
                scale = (x64.pow(2).sum(2) / D + EPS).pow(-0.5).view(H, N, 1)
                gain = w.double().view(1, 1, D)
            else:
                scale, gain = 1.0, 1.0
            src = x64 * scale * gain if dy is None else dy[i].double()
            z = torch.complex(src[..., lo], src[..., hi]) * (factor if dy is None else factor.conj())
            res = torch.empty_like(src)
            res[..., lo], res[..., hi] = z.real, z.imag
            if dy is not None and case["norm"] != "none":
                dw += (res * x64 * scale).sum(1)
                up = res * gain
                dot = (up * x64).sum((0, 2), keepdim=True) / (H * D) if case["norm"] == "token" else (up * x64).sum(2, keepdim=True) / D
                res = scale * up - x64 * scale ** 3 * dot
            out[i] = res
        if dy is None or case["norm"] == "none":
            return out, None
        return out, dw.flatten() if case["norm"] == "token" else dw.sum(0)

    if case["pass"] == "fwd":
        return {"q": one(s["q"], s["qw"], None)[0], "k": one(s["k"], s["kw"], None)[0]}
    (dq, dqw), (dk, dkw) = one(s["q"], s["qw"], s["dq_out"]), one(s["k"], s["kw"], s["dk_out"])
    return {"dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw}


def _exact_norm(case, s):
    M, K = case["tokens"], case["features"]
    w = s["w"].double()
    if case["pass"] == "bwd":
        dx, dw = torch.empty((M, K), dtype=torch.float64, device="cuda"), torch.zeros(K, dtype=torch.float64, device="cuda")
        for r0 in range(0, M, 8192):
            r1 = min(M, r0 + 8192)
            x, dy = s["x"][r0:r1].double(), s["dy"][r0:r1].double()
            inv = 1.0 / torch.sqrt(x.pow(2).sum(1, keepdim=True) / K + EPS)
            dw += (dy * x * inv).sum(0)
            up = dy * w
            dx[r0:r1] = up * inv - x * inv ** 3 * (up * x).sum(1, keepdim=True) / K
            if s["res"] is not None:
                dx[r0:r1] += s["res"][r0:r1].double()
        return {"dx": dx, "dw": dw}
    h = s["x"].clone()
    y = torch.empty((M, case["outputs"] or K), dtype=torch.float64, device="cuda")
    weight = s["weight"].double() if case["pass"] == "linear" else None
    for r0 in range(0, M, 8192):                 # (whole blocks of 128 tokens)
        r1 = min(M, r0 + 8192)
        if s["res"] is not None:
            h[r0:r1] = (s["x"][r0:r1].double() + s["res"][r0:r1].double()).bfloat16()
        x = h[r0:r1].double()
        n = x / torch.sqrt(x.pow(2).sum(1, keepdim=True) / K + EPS) * w
        if weight is None:
            y[r0:r1] = n
            continue
        for b0 in range(0, r1 - r0, 128):
            part = n[b0:b0 + 128]
            top = part.abs().amax(0).view(K // 128, 128).amax(1)
            step = torch.where(top > 0, top / 127.0, torch.ones_like(top)).repeat_interleave(128)
            n[b0:b0 + 128] = torch.round(part / step) * step
        y[r0:r1] = n @ weight.t()
        if s["bias"] is not None:
            y[r0:r1] += s["bias"].double()
    return {"y": y, "h": h}


def _exact_cross(case, s):
    B, H, G, lens = case["batch"], case["heads"], case["kv_heads"], _lens(case)
    out = torch.zeros((B, H, case["queries"], D), dtype=torch.float64, device="cuda")
    train = case["pass"] == "train"
    dq = torch.zeros_like(out) if train else None
    dk, dv = [torch.zeros((B, G, case["keys"], D), dtype=torch.float64, device="cuda") for _ in range(2)] if train else (None, None)
    scale = D ** -0.5
    for i in range(B):
        if lens[i] == 0:
            continue                             # nothing to attend to: zeros
        for h in range(H):
            g = h // (H // G)
            q, k, v = s["q"][i, h].double(), s["k"][i, g, :lens[i]].double(), s["v"][i, g, :lens[i]].double()
            p = torch.softmax(q @ k.t() * scale, 1)
            out[i, h] = p @ v
            if train:
                do = s["dout"][i, h].double()
                dp = do @ v.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
                dq[i, h] = ds @ k
                dk[i, g, :lens[i]] += ds.t() @ q
                dv[i, g, :lens[i]] += p.t() @ do
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if train else {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "norm": _exact_norm, "cross": _exact_cross}[case["family"]](case, s)
