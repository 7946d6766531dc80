"""What a model does next with looked-up rows, as timed passes: a learned position bias by buckets and its
gradient, dropout from a counter-based generator, and the join at which a block's output enters the rows again
(norms before and after, gate, residual scale), forward and backward.

A pass is one public call on buffers that the caller keeps.  With `own` false the same outputs come from
elementary torch operations in 32 bits (64 for long sums); `exact` gives them from the definitions in 64 bits.
"""
import bisect
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases


def _bias(name, do, N, H, Q, K, dtype, buckets=32, far=128, two_sided=False, causal=False, starts=False):
    """do: "bias" (the bias itself) or "bias_grad" (gradient of the bucket rows).
    starts: every sequence has its own position of the first query (a batch of caches of different lengths);
    else the last query stands at the last key (one position for all)."""
    return dict(name=name, do=do, N=N, H=H, Q=Q, K=K, dtype=dtype, buckets=buckets, far=far, two_sided=two_sided,
                causal=causal, starts=starts)


def _dropout(name, rows, d, dtype, p=0.1):
    return dict(name=name, do="dropout", rows=rows, d=d, dtype=dtype, p=p)


def _join(name, do, rows, d, dtype, norm, gate, p=0.0, scale=1.0, post=True, pre=True):
    """do: "join" or "join_grad".  gate: "none", "row" (one number per row), "element" (one per element) or a
    number g as text: a vector per g rows.  post, pre: norm of the block's output, norm of the sum."""
    return dict(name=name, do=do, rows=rows, d=d, dtype=dtype, norm=norm, gate=gate, p=p, scale=scale, post=post,
                pre=pre)


def listed():
    return [
        # one new token of one sequence, full-precision bias: as small as the call gets, latency counts
        _bias("bias_token", "bias", 1, 16, 1, 1024, "f32", causal=True),
        # one new token of each of 64 sequences of different lengths, odd cache length
        _bias("bias_serve", "bias", 64, 16, 1, 8191, "bf16", causal=True, starts=True),
        # the bias of a two-sided attention of 2048 positions, shared by the batch
        _bias("bias_2048", "bias", 1, 16, 2048, 2048, "bf16", two_sided=True),
        # training on ragged lengths: rows of an odd number of keys, later positions masked
        _bias("bias_grad_odd", "bias_grad", 4, 12, 777, 1001, "bf16", causal=True),
        # a training step's largest: the gradient of a broadcast bias, 16 sequences of 2048
        _bias("bias_grad_2048", "bias_grad", 16, 16, 2048, 2048, "bf16", two_sided=True),
        # dropout on the rows of a small lookup: 256 samples of 26 fields of 16
        _dropout("dropout_small", 256 * 26, 16, "f32"),
        # dropout on the rows of a training lookup of the 100 MB model
        _dropout("dropout_large", 32_768 * 26, 128, "bf16"),
        # one new token of each of 16 sequences through the join of a wide model
        _join("join_token", "join", 16, 4096, "bf16", "rms", "none", scale=0.5),
        # rows of a ranker: every field's row normed and gated by its own number, normed again for the next layer
        _join("join_fields", "join", 8192 * 26, 128, "f32", "layer", "row"),
        # the join behind a block of a wide sequence model in training: gate per element, dropout
        _join("join_block", "join", 16_384, 4096, "bf16", "rms", "element", p=0.1, scale=0.5),
        # gradients of the ranker's rows, d no power of two
        _join("join_grad_fields", "join_grad", 8192 * 26, 100, "f32", "layer", "row"),
        # gradients of the wide model's join, a gate vector per sequence of 1024
        _join("join_grad_block", "join_grad", 16_384, 4096, "bf16", "rms", "1024", p=0.1, scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    do = rng.choice(["bias", "bias", "bias_grad", "bias_grad", "dropout", "join", "join", "join_grad", "join_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if do.startswith("bias"):
        two_sided = rng.random() < 0.5
        buckets = 2 * rng.randint(4, 32)
        far = rng.randint(buckets, 16 * buckets)
        H = rng.randint(1, 32)
        serve = do == "bias" and rng.random() < 0.4
        if serve:
            N, Q, K = _log_int(rng, 1, 64), 1, _log_int(rng, 64, 32_768)
        else:
            N = 1 if do == "bias" else _log_int(rng, 1, 16)
            Q, K = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        while N * H * Q * K > 1 << 29:
            H = max(1, H // 2)
        return _bias("", do, N, H, Q, K, dtype, buckets, far, two_sided, rng.random() < 0.5, N > 1 and rng.random() < 0.5)
    if do == "dropout":
        d = _log_int(rng, 3, 4096)
        rows = _log_int(rng, 1, max(2, min(1_000_000, (1 << 27) // d)))
        return _dropout("", rows, d, dtype, rng.choice([0.05, 0.1, 0.2, 0.5]))
    d = _log_int(rng, 8, 8192)
    if rng.random() < 0.5:
        d = max(8, d // 8 * 8)
    rows = _log_int(rng, 1, max(2, min(500_000, (1 << 26) // d)))
    gate = rng.choice(["none", "row", "element", "group"])
    if gate == "group":
        g = _log_int(rng, 2, 1024)
        rows = max(1, rows // g) * g
        while rows * d > 1 << 26:
            rows -= g
        if rows < g:
            g = rows = max(2, (1 << 26) // d // 2)
        gate = str(g)
    post = rng.random() < 0.8
    return _join("", do, rows, d, dtype, rng.choice(["rms", "layer"]), gate, rng.choice([0.0, 0.1]),
                 rng.choice([1.0, 0.5]), post, not post or rng.random() < 0.8)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    do = case["do"]
    if do.startswith("bias"):
        n = case["N"] * case["H"] * case["Q"] * case["K"]
        return {"bytes": e * n + 4 * case["buckets"] * case["H"], "flops": n if do == "bias_grad" else 0}
    n = case["rows"] * case["d"]
    if do == "dropout":
        return {"bytes": 2 * e * n, "flops": n}
    gate, groups = _gate_shape(case)
    gate_n = gate[0] * gate[1] if gate else 0
    weights = (int(case["post"]) + int(case["pre"])) * case["d"] * 4
    if do == "join":
        return {"bytes": e * (n * (3 + int(case["pre"])) + gate_n) + weights, "flops": 12 * n}
    return {"bytes": e * (n * (4 + 2 * int(case["pre"])) + 2 * gate_n) + 2 * weights, "flops": 30 * n}


def _gate_shape(case):
    g = case["gate"]
    if g == "none":
        return None, 0
    if g == "row":
        return (case["rows"], 1), 1
    if g == "element":
        return (case["rows"], case["d"]), 1
    return (case["rows"] // int(g), case["d"]), int(g)


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    do = case["do"]
    s = {"case": case}
    if do.startswith("bias"):
        N, H, Q, K = case["N"], case["H"], case["Q"], case["K"]
        s["q_start"] = K - Q
        if case["starts"]:  # sequences of different lengths, the new tokens at their ends
            lengths = torch.randint(max(1, K // 8), K + 1, (N,), generator=gen, device=dev)
            s["q_start"] = (lengths - Q).contiguous()
        if do == "bias":
            s["rows"] = normal(case["buckets"], H, scale=0.5)
            if own:
                s["out"] = torch.empty(N, H, Q, K, dtype=dt, device=dev)
        else:
            # gradients of attention scores: a probability's share, both signs
            s["grad"] = torch.empty(N, H, Q, K, dtype=dt, device=dev)
            for n in range(N):
                s["grad"][n] = normal(H, Q, K, scale=1.0 / K, dtype=dt)
            if own:
                s["grad_rows"] = torch.empty(case["buckets"], H, device=dev)
        if own:
            import paper_2108_02191_b200 as robe
            s["bias"] = robe.robe_bias_create(case["buckets"], case["far"], case["two_sided"])
            if do == "bias_grad":
                s["workspace"] = torch.empty(robe.robe_bias_backward_workspace_bytes(s["bias"], H, N, Q, K),
                                             dtype=torch.uint8, device=dev)
        return s

    rows, d = case["rows"], case["d"]
    s["seed"] = int(torch.randint(1 << 60, (1,), generator=gen, device=dev).item())
    s["offset"] = 7 * seed + 1
    s["step"] = torch.randint(1 << 40, (1,), generator=gen, device=dev)  # a training loop's counter, on the device
    if do == "dropout":
        s["x"] = normal(rows, d, scale=0.05, dtype=dt)
        if own:
            s["out"] = torch.empty_like(s["x"])
        return s
    s["x"] = normal(rows, d, scale=0.7, dtype=dt)
    s["w_post"] = 1.0 + normal(d, scale=0.1) if case["post"] else None
    s["w_pre"] = 1.0 + normal(d, scale=0.1) if case["pre"] else None
    shape, _ = _gate_shape(case)
    s["gate"] = torch.sigmoid(normal(*shape)).to(dt) if shape else None
    if do == "join":
        s["residual"] = normal(rows, d, scale=1.5, dtype=dt)
        if own:
            s["out"] = torch.empty_like(s["x"])
            s["normed"] = torch.empty_like(s["x"]) if case["pre"] else None
        return s
    s["out"] = normal(rows, d, scale=1.7, dtype=dt) if case["pre"] else None  # as the forward call stored it
    s["grad_out"] = normal(rows, d, scale=0.01, dtype=dt)
    s["grad_normed"] = normal(rows, d, scale=0.01, dtype=dt) if case["pre"] else None
    if own:
        import paper_2108_02191_b200 as robe
        s["grad_x"] = torch.empty_like(s["x"])
        s["grad_residual"] = torch.empty_like(s["x"])
        s["grad_gate"] = torch.empty_like(s["gate"]) if shape else None
        s["grad_w_post"] = torch.empty(d, device=dev) if case["post"] else None
        s["grad_w_pre"] = torch.empty(d, device=dev) if case["pre"] else None
        s["workspace"] = torch.empty(robe.robe_residual_backward_workspace_bytes(rows, d, shape[0] if shape else 0),
                                     dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    do = case["do"]
    if not own:
        return {"bias": _plain_bias, "bias_grad": _plain_bias_grad, "dropout": _plain_dropout, "join": _plain_join,
                "join_grad": _plain_join_grad}[do](s)
    import paper_2108_02191_b200 as robe
    if do == "bias":
        robe.robe_bias_forward(s["bias"], s["rows"], s["out"], s["q_start"], case["causal"])
        return s["out"]
    if do == "bias_grad":
        robe.robe_bias_backward(s["bias"], s["grad"], s["grad_rows"], s["workspace"], s["q_start"], case["causal"])
        return s["grad_rows"]
    if do == "dropout":
        robe.robe_dropout(s["x"], s["out"], case["p"], s["seed"], s["offset"], s["step"])
        return s["out"]
    norm = robe.ROBE_NORM_RMS if case["norm"] == "rms" else robe.ROBE_NORM_LAYER
    step = s["step"] if case["p"] else None
    if do == "join":
        robe.robe_residual_forward(s["x"], s["residual"], s["out"], s["normed"], s["w_post"], s["w_pre"], s["gate"],
                                   case["scale"], norm, EPS, case["p"], s["seed"], s["offset"], step)
        return [s["out"], s["normed"]] if case["pre"] else [s["out"]]
    robe.robe_residual_backward(s["grad_out"], s["grad_normed"], s["x"], s["out"], s["grad_x"], s["grad_residual"],
                                s["w_post"], s["w_pre"], s["gate"], s["grad_w_post"], s["grad_w_pre"], s["grad_gate"],
                                s["workspace"], case["scale"], norm, EPS, case["p"], s["seed"], s["offset"], step)
    return [g for g in (s["grad_x"], s["grad_residual"], s["grad_gate"], s["grad_w_post"], s["grad_w_pre"])
            if g is not None]


EPS = 1e-6

# ---- plain forms: position bias


def _edges(case):
    """Smallest distance of every bucket of one side: the first half exact, then powers of (far / half)."""
    side = case["buckets"] // 2 if case["two_sided"] else case["buckets"]
    half = side // 2
    edges = list(range(half))
    steps = side - half
    for k in range(steps):
        n = max(half, int(half * (case["far"] / half) ** (k / steps)) - 2)
        while n ** steps < half ** (steps - k) * case["far"] ** k:
            n += 1
        edges.append(n)
    return edges


def _distances(s):
    """Key position minus query position: [N or 1, Q, K]."""
    case = s["case"]
    dev = torch.device("cuda")
    q = torch.arange(case["Q"], device=dev)
    start = s["q_start"] if torch.is_tensor(s["q_start"]) else torch.tensor([s["q_start"]], device=dev)
    q = start[:, None, None] + q[None, :, None]
    return torch.arange(case["K"], device=dev)[None, None, :] - q


def _buckets(case, r):
    edges = torch.tensor(_edges(case)[1:], device=r.device)
    if case["two_sided"]:
        dist = r.abs()
        return torch.bucketize(dist, edges, right=True) + torch.where(r > 0, case["buckets"] // 2, 0)
    return torch.bucketize((-r).clamp(min=0), edges, right=True)


def _plain_bias(s):
    case = s["case"]
    r = _distances(s)
    b = s["rows"][_buckets(case, r)]  # [N or 1, Q, K, H]
    if case["causal"]:
        b = torch.where((r > 0)[..., None], -math.inf, b)
    b = b.permute(0, 3, 1, 2)
    return b.expand(case["N"], -1, -1, -1).to(DTYPES[case["dtype"]]).contiguous()


def _plain_bias_grad(s):
    case = s["case"]
    r = _distances(s)
    bucket = _buckets(case, r)
    if case["causal"]:
        bucket = torch.where(r > 0, -1, bucket)
    out = torch.zeros(case["buckets"], case["H"], dtype=torch.float64, device="cuda")
    for n in range(case["N"]):
        g = s["grad"][n].float()
        of = bucket[n if bucket.shape[0] > 1 else 0]
        for b in range(case["buckets"]):
            out[b] += torch.where(of == b, g, 0.0).sum((1, 2), dtype=torch.float64)
    return out.float()


# ---- plain forms: dropout.  Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
# easy as 1, 2, 3", 2011), in 64-bit integers


def _mul_hi_lo(m, c):
    t = m * (c & 0xFFFF)
    u = m * (c >> 16) + (t >> 16)
    return u >> 16, ((u & 0xFFFF) << 16) | (t & 0xFFFF)


def _plain_keep(s, rows, d):
    """Truth per element: kept.  Element (r, c) goes by 16-bit half c mod 8 of the words of counter (c / 8, r, offset)."""
    dev = torch.device("cuda")
    off = s["step"][0] + s["offset"]
    groups = (d + 7) // 8
    c0 = torch.arange(groups, device=dev)[None, :].expand(rows, groups)
    c1 = torch.arange(rows, device=dev)[:, None].expand(rows, groups)
    c2 = (off & 0xFFFFFFFF).expand(rows, groups)
    c3 = ((off >> 32) & 0xFFFFFFFF).expand(rows, groups)
    k0, k1 = s["seed"] & 0xFFFFFFFF, (s["seed"] >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mul_hi_lo(0xD2511F53, c0)
        h1, l1 = _mul_hi_lo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    return words.reshape(rows, groups * 8)[:, :d] >= _threshold(s["case"]["p"])


def _threshold(p):
    return int(math.floor(float(np.float32(p)) * 65536 + 0.5))


def _drop(s, v):
    p = s["case"]["p"]
    if p == 0.0:
        return v
    return torch.where(_plain_keep(s, *v.shape), v * (65536.0 / (65536 - _threshold(p))), 0.0)


def _plain_dropout(s):
    return _drop(s, s["x"].float()).to(s["x"].dtype)


# ---- plain forms: join


def _norm(case, v):
    if case["norm"] == "layer":
        v = v - v.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * rstd, rstd


def _norm_grad(case, n, rstd, v):
    v = v - n * (v * n).mean(-1, keepdim=True) if case["norm"] == "rms" else \
        v - v.mean(-1, keepdim=True) - n * (v * n).mean(-1, keepdim=True)
    return v * rstd


def _spread(case, gate):
    gate = gate.float()
    _, per = _gate_shape(case)
    return gate.repeat_interleave(per, 0) if per > 1 else gate


def _plain_join(s):
    case = s["case"]
    y = s["x"].float()
    if case["post"]:
        y = _norm(case, y)[0] * s["w_post"]
    y = _drop(s, y) * case["scale"]
    if s["gate"] is not None:
        y = y * _spread(case, s["gate"])
    out = s["residual"].float() + y
    dt = s["x"].dtype
    if not case["pre"]:
        return [out.to(dt)]
    return [out.to(dt), (_norm(case, out)[0] * s["w_pre"]).to(dt)]


def _plain_join_grad(s):
    case = s["case"]
    dt = s["x"].dtype
    t = s["grad_out"].float()
    grads = {}
    if case["pre"]:
        n, rstd = _norm(case, s["out"].float())
        gn = s["grad_normed"].float()
        grads["w_pre"] = (gn * n).sum(0, dtype=torch.float64).float()
        t = t + _norm_grad(case, n, rstd, gn * s["w_pre"])
    y = s["x"].float()
    if case["post"]:
        n, rstd = _norm(case, y)
        y = n * s["w_post"]
    u = t * case["scale"]
    if s["gate"] is not None:
        g = _drop(s, y) * u
        shape, per = _gate_shape(case)
        if case["gate"] == "row":
            g = g.sum(1, keepdim=True)
        elif per > 1:
            g = g.reshape(shape[0], per, shape[1]).sum(1, dtype=torch.float64)
        grads["gate"] = g.to(dt)
        u = u * _spread(case, s["gate"])
    u = _drop(s, u)
    if case["post"]:
        grads["w_post"] = (u * n).sum(0, dtype=torch.float64).float()
        u = _norm_grad(case, n, rstd, u * s["w_post"])
    order = [u.to(dt), t.to(dt), grads.get("gate"), grads.get("w_post"), grads.get("w_pre")]
    return [g for g in order if g is not None]


# ---------------------------------------------------------------- 64 bits, from the definitions


def exact(case, seed):
    s = prepare(case, seed)
    return {"bias": _exact_bias, "bias_grad": _exact_bias_grad, "dropout": _exact_dropout, "join": _exact_join,
            "join_grad": _exact_join_grad}[case["do"]](s)


def _bucket_of_diagonals(case, first, count):
    """Buckets of the distances first .. first + count - 1 (key minus query), -1 where masked; Python integers."""
    side = case["buckets"] // 2 if case["two_sided"] else case["buckets"]
    half, far = side // 2, case["far"]
    steps = side - half
    reached = [half ** (steps - k) * far ** k for k in range(steps)]  # dist ** steps has to reach these

    def of(r):
        if r > 0 and case["causal"]:
            return -1
        n = abs(r) if case["two_sided"] else max(-r, 0)
        b = n if n < half else side - 1 if n >= far else half + bisect.bisect_right(reached, n ** steps) - 1
        return b + (side if case["two_sided"] and r > 0 else 0)

    return np.array([of(r) for r in range(first, first + count)], dtype=np.int64)


def _starts(s):
    if torch.is_tensor(s["q_start"]):
        return [int(v) for v in s["q_start"].tolist()]
    return [s["q_start"]] * s["case"]["N"]


def _exact_bias(s):
    case = s["case"]
    N, H, Q, K = case["N"], case["H"], case["Q"], case["K"]
    out = torch.empty(N, H, Q, K, dtype=torch.float64, device="cuda")
    rows = torch.cat([s["rows"].double(), torch.full((1, H), -math.inf, dtype=torch.float64, device="cuda")])
    for n, start in enumerate(_starts(s)):
        # diagonal i - j = const holds one value: row i is the window of the diagonals that starts at Q - 1 - i
        b = torch.from_numpy(_bucket_of_diagonals(case, -(Q - 1) - start, Q + K - 1)).cuda()
        out[n] = rows[b].t().unfold(1, K, 1).flip(1)
    return out


def _exact_bias_grad(s):
    case = s["case"]
    H, Q, K = case["H"], case["Q"], case["K"]
    out = torch.zeros(case["buckets"] + 1, H, dtype=torch.float64, device="cuda")
    for n, start in enumerate(_starts(s)):
        b = torch.from_numpy(_bucket_of_diagonals(case, -(Q - 1) - start, Q + K - 1)).cuda()
        b = torch.where(b < 0, case["buckets"], b)
        # rows laid one place further right each, from the last up: columns are then the diagonals
        wide = torch.zeros(H, Q, Q + K, dtype=torch.float64, device="cuda")
        wide[:, :, :K] = s["grad"][n].double().flip(1)
        diagonals = wide.reshape(H, -1)[:, :Q * (Q + K - 1)].reshape(H, Q, Q + K - 1).sum(1)
        out.index_add_(0, b, diagonals.t())
    return out[:-1]


def _exact_keep(s, rows, d):
    """Kept elements, numpy, a row block at a time."""
    off = (int(s["step"].item()) + s["offset"]) % (1 << 64)
    groups = -(-d // 8)
    out = np.empty((rows, d), dtype=bool)
    low, t = np.uint64(0xFFFFFFFF), _threshold(s["case"]["p"])
    block = max(1, (1 << 20) // groups)
    for a in range(0, rows, block):
        n = min(block, rows - a)
        c = [np.tile(np.arange(groups, dtype=np.uint64), (n, 1)),
             np.tile(np.arange(a, a + n, dtype=np.uint64)[:, None], (1, groups)),
             np.full((n, groups), off & 0xFFFFFFFF, dtype=np.uint64), np.full((n, groups), off >> 32, dtype=np.uint64)]
        key = [s["seed"] & 0xFFFFFFFF, s["seed"] >> 32]
        for _ in range(10):
            p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), p1 & low,
                 (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), p0 & low]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        words = np.stack(c, -1).astype(np.uint32).view(np.uint16)  # low half first
        out[a:a + n] = (words.reshape(n, groups * 8) >= t)[:, :d]
    return torch.from_numpy(out).cuda()


def _exact_factor(s, rows, d):
    """What dropout multiplies by, per element."""
    p = s["case"]["p"]
    if p == 0.0:
        return 1.0
    return _exact_keep(s, rows, d).double() * (65536.0 / (65536 - _threshold(p)))


def _exact_dropout(s):
    return s["x"].double() * _exact_factor(s, *s["x"].shape)


def _exact_norm(case, v):
    mean = v.mean(1, keepdim=True) if case["norm"] == "layer" else torch.zeros_like(v[:, :1])
    return (v - mean) / (((v - mean) ** 2).mean(1, keepdim=True) + EPS).sqrt()


def _exact_gate(s):
    case = s["case"]
    if s["gate"] is None:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda")
    g = s["gate"].double()
    per = case["rows"] // g.shape[0]
    return g[:, None, :].expand(-1, per, -1).reshape(case["rows"], g.shape[1])


def _exact_join(s):
    case = s["case"]
    x = s["x"].double()
    y = _exact_norm(case, x) * s["w_post"].double() if case["post"] else x
    out = s["residual"].double() + y * _exact_factor(s, *x.shape) * _exact_gate(s) * case["scale"]
    return [out, _exact_norm(case, out) * s["w_pre"].double()] if case["pre"] else [out]


def _exact_join_grad(s):
    """By the chain rule through the forward formula, torch's derivatives in 64 bits."""
    case = s["case"]
    rows, d = case["rows"], case["d"]
    factor = _exact_factor(s, rows, d)
    x = s["x"].double().requires_grad_()
    w_post = s["w_post"].double().requires_grad_() if case["post"] else None
    t = s["grad_out"].double()
    w_pre_grad = None
    if case["pre"]:
        out = s["out"].double().requires_grad_()
        w_pre = s["w_pre"].double().requires_grad_()
        normed = _exact_norm(case, out) * w_pre
        through, w_pre_grad = torch.autograd.grad(normed, [out, w_pre], s["grad_normed"].double())
        t = t + through
    y = _exact_norm(case, x) * w_post if case["post"] else x
    y = y * factor * case["scale"]
    leaves = [x] + ([w_post] if case["post"] else [])
    if s["gate"] is not None:
        gate = s["gate"].double().requires_grad_()
        per = rows // gate.shape[0]
        y = y * gate[:, None, :].expand(-1, per, -1).reshape(rows, gate.shape[1])
        leaves.append(gate)
    else:
        y = y * 1.0
    got = list(torch.autograd.grad(y, leaves, t))
    order = [got[0], t, got[-1] if s["gate"] is not None else None, got[1] if case["post"] else None, w_pre_grad]
    return [g for g in order if g is not None]
