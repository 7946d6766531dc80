"""Rows of plain tables and rows in 8 bits, as timed passes: the lookup in an uncompressed table with scaling and its
gradient by sorted ids; the join of a block's output with the residual whose norm leaves as 8-bit codes with scales; a
paged cache of rows that is quantised as it is written, and read back; and the attention of one new token over two such
caches, with the learned position bias.

A pass is one public call on buffers that the caller keeps.  With `own` false the same outputs come from elementary
torch operations in 32 bits (64 for long sums); `exact` gives them from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
LARGEST = {"e4m3": 448.0, "i8": 127.0}
SMALLEST = 2.0 ** -90  # groups whose values are all smaller are scaled as if this were their largest
EPS = 1e-6


# ---------------------------------------------------------------- cases


def _table(name, do, n, V, d, table, rows, ids="i64", zipf=True, accumulate=False, scale=1.0):
    """do: "lookup" or "table_grad".  n ids into V rows of d; table, rows: types of the table and of the rows (of the
    gradient rows: the table's gradient is fp32).  zipf: ids follow Zipf(1.05) (frequent ones first), else uniform.
    accumulate: the gradient is added to what is there, else every row of it is written."""
    return dict(name=name, do=do, n=n, V=V, d=d, table=table, rows=rows, ids=ids, zipf=zipf, accumulate=accumulate, scale=scale)


def _join8(name, rows, d, dtype, group, norm="rms", scale=1.0, residual=True):
    """group: columns that share a scale, 0 for the whole row.  residual False: nothing is added to (a model's entry)."""
    return dict(name=name, do="join8", rows=rows, d=d, dtype=dtype, group=group, norm=norm, scale=scale, residual=residual)


def _cache(name, do, N, new, past, heads, dim, dtype, code, page, ragged):
    """do: "cache_write" or "cache_read".  N sequences of `new` rows (ragged: of 1 .. new, packed) behind up to `past` rows
    that are there already; a row is heads x dim with a scale for each head; pages of `page` rows."""
    return dict(name=name, do=do, N=N, new=new, past=past, heads=heads, dim=dim, dtype=dtype, code=code, page=page, ragged=ragged)


def _attend(name, N, most, heads, group, dim, code, page, buckets=0, far=128):
    """N sequences, each with one new token (the last of its up to `most` rows in the caches of keys and values): heads x group
    query heads over `heads` of the cache; buckets: of the position bias' distances, 0 for none."""
    return dict(name=name, do="attend", N=N, most=most, heads=heads, group=group, dim=dim, code=code, page=page, buckets=buckets, far=far)


def listed():
    return [
        # one new token of each of 16 sequences: as small as the lookup gets, latency counts
        _table("lookup_token", "lookup", 16, 65_536, 4096, "bf16", "bf16", scale=64.0),
        # a ranker's training lookup in a table that is not compressed: fp32 weights, bf16 rows
        _table("lookup_fields", "lookup", 32_768 * 26, 1_000_000, 128, "f32", "bf16"),
        # the wide sequence model's gradient, added to what the output layer has left in the same matrix
        _table("table_grad_tokens", "table_grad", 16_384, 65_536, 4096, "f32", "bf16", accumulate=True, scale=64.0),
        # the ranker's gradient, every row of it written
        _table("table_grad_fields", "table_grad", 32_768 * 26, 1_000_000, 64, "f32", "f32"),
        # odd sizes, 32-bit ids, rows that are not of whole 16-byte pieces
        _table("table_grad_odd", "table_grad", 5003, 32_003, 1001, "f32", "bf16", ids="i32"),
        # one new token of each of 16 sequences through the join, a scale per 128 columns
        _join8("join8_token", 16, 4096, "bf16", 128),
        # the wide model's training step
        _join8("join8_block", 16_384, 4096, "bf16", 128),
        # one new token's keys of each of 64 sequences of different lengths
        _cache("cache_write_token", "cache_write", 64, 1, 2047, 8, 128, "bf16", "e4m3", 64, False),
        # prompts of different lengths, packed
        _cache("cache_write_prompts", "cache_write", 16, 4096, 0, 8, 128, "bf16", "e4m3", 64, True),
        # what 64 sequences have in the cache, for an attention that takes rows as they are
        _cache("cache_read", "cache_read", 64, 4096, 0, 8, 128, "bf16", "e4m3", 64, True),
        # a serving step: one new token of each of 64 sequences of different lengths, grouped heads, position bias
        _attend("attend_serve", 64, 8191, 8, 4, 128, "e4m3", 64, buckets=32),
        # one sequence alone, long: work has to be split over its length
        _attend("attend_one", 1, 65_521, 4, 8, 128, "e4m3", 64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    do = rng.choice(["lookup", "table_grad", "table_grad", "join8", "join8", "cache_write", "cache_read", "attend", "attend"])
    if do in ("lookup", "table_grad"):
        d = _log_int(rng, 8, 8192)
        if rng.random() < 0.6:
            d = max(8, d // 8 * 8)
        V = _log_int(rng, 100, max(200, min(4_000_000, (1 << 26) // d)))
        n = _log_int(rng, 1, max(2, min(1_000_000, (1 << 25) // d)))
        rows = rng.choice(["f32", "bf16"])
        table = rng.choice(["f32", "bf16"]) if do == "lookup" else "f32"
        return _table("", do, n, V, d, table, rows, rng.choice(["i64", "i32"]), rng.random() < 0.6, do == "table_grad" and rng.random() < 0.5,
                      rng.choice([1.0, math.sqrt(d), 0.125]))
    if do == "join8":
        d = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            d = max(16, d // 8 * 8)
        rows = _log_int(rng, 1, max(2, min(400_000, (1 << 25) // d)))
        return _join8("", rows, d, rng.choice(["f32", "bf16"]), rng.choice([0, 32, 64, 128]), rng.choice(["rms", "rms", "layer"]),
                      rng.choice([1.0, 0.5]), rng.random() < 0.8)
    heads, dim, page = rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 80, 96, 128, 256]), rng.choice([16, 32, 64, 128])
    N = _log_int(rng, 1, 64)
    if do == "attend":
        dim = rng.choice([64, 96, 128, 256])
        most = _log_int(rng, 1, max(2, min(65_536, (1 << 28) // (N * heads * dim))))
        return _attend("", N, most, heads, rng.choice([1, 2, 4, 5, 8, 16]), dim, rng.choice(["e4m3", "i8"]), page, rng.choice([0, 32, 64]),
                       rng.choice([128, 512]))
    most = max(2, min(8192, (1 << 26) // (N * heads * dim)))
    new = 1 if do == "cache_write" and rng.random() < 0.4 else _log_int(rng, 2, most)
    past = rng.randint(0, min(2048, most)) if do == "cache_write" else 0
    return _cache("", do, N, new, past, heads, dim, rng.choice(["f32", "bf16"]), rng.choice(["e4m3", "i8"]), page,
                  new > 1 and rng.random() < 0.7)


def _zipf_weights(V, device):
    w = torch.arange(1, V + 1, dtype=torch.float64, device=device) ** -1.05
    return w / w.sum()


def _distinct(case):
    """Expected number of different rows among the ids."""
    n, V = case["n"], case["V"]
    if not case["zipf"]:
        return V * -math.expm1(n * math.log1p(-1.0 / V))
    return float(-torch.expm1(n * torch.log1p(-_zipf_weights(V, "cpu"))).sum())


def _lengths(case):
    """Rows of every sequence, spread over the range; which sequence has which goes by the inputs."""
    N = case["N"]
    if case["do"] == "attend":
        low, high = max(1, case["most"] // 8), case["most"]
    else:
        low, high = 1 if case["ragged"] else case["new"], case["new"]
    return [low + round((high - low) * (0.618034 * (k + 1) % 1.0)) if N > 1 else high for k in range(N)]


def work(case):
    do = case["do"]
    size = {"f32": 4, "bf16": 2, "i64": 8, "i32": 4}
    if do in ("lookup", "table_grad"):
        n, d = case["n"], case["d"]
        read = n * size[case["ids"]]
        if do == "lookup":
            return {"bytes": read + int(_distinct(case) * d) * size[case["table"]] + n * d * size[case["rows"]], "flops": n * d}
        wrote = int(_distinct(case) * d) * 8 if case["accumulate"] else case["V"] * d * 4
        return {"bytes": read + n * d * size[case["rows"]] + wrote, "flops": n * d}
    if do == "join8":
        n = case["rows"] * case["d"]
        groups = case["rows"] * (-(-case["d"] // case["group"]) if case["group"] else 1)
        return {"bytes": n * (size[case["dtype"]] * (3 if case["residual"] else 2) + 1) + 4 * (groups + case["d"]), "flops": 10 * n}
    if do == "attend":
        keys, q = sum(_lengths(case)) * case["heads"], case["N"] * case["heads"] * case["group"]
        return {"bytes": keys * 2 * (case["dim"] + 4) + q * case["dim"] * 4 + case["buckets"] * case["heads"] * case["group"] * 4,
                "flops": keys * case["group"] * case["dim"] * 4}
    rows = sum(_lengths(case))
    n = rows * case["heads"] * case["dim"]
    return {"bytes": int(n * (size[case["dtype"]] + 1) + 4 * rows * case["heads"]), "flops": int(2 * n)}


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    def ints(lo, hi, n):
        return torch.randint(lo, hi + 1, (n,), generator=gen, device=dev)

    do = case["do"]
    s = {"case": case}
    if do in ("lookup", "table_grad"):
        n, V, d = case["n"], case["V"], case["d"]
        if case["zipf"]:
            edges = _zipf_weights(V, dev).cumsum(0)
            ids = torch.bucketize(torch.rand(n, generator=gen, device=dev, dtype=torch.float64), edges).clamp_(max=V - 1)
        else:
            ids = ints(0, V - 1, n)
        s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        rows = DTYPES[case["rows"]]
        if do == "lookup":
            s["table"] = normal(V, d, scale=0.02, dtype=DTYPES[case["table"]])
            s["out"] = torch.empty(n, d, dtype=rows, device=dev)
        else:
            s["grad"] = normal(n, d, scale=0.01, dtype=rows)
            s["grad_table"] = normal(V, d, scale=0.01)  # accumulating: what the output layer has left there
        if do == "table_grad" and own:
            import paper_2108_02191_b200 as robe
            s["workspace"] = torch.empty(robe.robe_table_backward_workspace_bytes(n, V, d), dtype=torch.uint8, device=dev)
        return s
    if do == "join8":
        rows, d, dt = case["rows"], case["d"], DTYPES[case["dtype"]]
        groups = -(-d // case["group"]) if case["group"] else 1
        s["x"] = normal(rows, d, scale=0.7, dtype=dt)
        s["residual"] = normal(rows, d, scale=1.5, dtype=dt) if case["residual"] else None
        s["w"] = 1.0 + normal(d, scale=0.1)
        s["out"] = torch.empty_like(s["x"])
        s["codes"] = torch.empty(rows, d, dtype=torch.float8_e4m3fn, device=dev)
        s["scales"] = torch.empty(rows, groups, device=dev)
        return s
    N, d, P = case["N"], case["heads"] * case["dim"], case["page"]
    lengths = torch.tensor(_lengths(case), device=dev)[torch.randperm(N, generator=gen, device=dev)]

    def codes(*shape):
        if case["code"] == "i8":
            return torch.randint(-127, 128, shape, generator=gen, device=dev, dtype=torch.int8)
        v = (normal(*shape) * 448.0 / 5.0).clamp_(-448.0, 448.0)
        return v.to(torch.float8_e4m3fn)

    if do == "attend":
        per = -(-case["most"] // P)
        s["pages"] = torch.randperm(N * per, generator=gen, device=dev).to(torch.int32).reshape(N, per)
        s["starts"] = lengths - 1  # where the new tokens stand
        s["q"] = normal(N, case["heads"] * case["group"], case["dim"], dtype=torch.bfloat16)
        spread = 5.0 if case["code"] == "e4m3" else 1.7
        for what in ("keys", "values"):
            s[what] = codes(N * per, P, d)
            s[what + "_scales"] = (0.5 + torch.rand(N * per, P, case["heads"], generator=gen, device=dev)) * spread / LARGEST[case["code"]]
        s["bias_rows"] = normal(case["buckets"], case["heads"] * case["group"], scale=0.5) if case["buckets"] else None
        s["out"] = torch.empty_like(s["q"])
        if own:
            import paper_2108_02191_b200 as robe
            s["bias"] = robe.robe_bias_create(case["buckets"], case["far"], False) if case["buckets"] else None
            s["workspace"] = torch.empty(robe.robe_cache_attention_workspace_bytes(N, case["heads"], case["heads"] * case["group"], case["dim"],
                                                                                   per * P), dtype=torch.uint8, device=dev)
        return s
    s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), lengths.cumsum(0)])
    s["starts"] = ints(0, case["past"], N) if case["past"] else torch.zeros(N, dtype=torch.int64, device=dev)
    total = sum(_lengths(case))
    per = -(-(case["past"] + case["new"]) // P)
    s["pages"] = torch.randperm(N * per, generator=gen, device=dev).to(torch.int32).reshape(N, per)
    if do == "cache_write":
        # keys: a few columns much larger than the others
        s["rows"] = (normal(total, d) * (1.0 + 9.0 * (torch.arange(d, device=dev) % 61 == 7))).to(DTYPES[case["dtype"]])
        s["codes"] = torch.zeros(N * per, P, d, dtype=torch.uint8, device=dev).view(CODES[case["code"]])
        s["scales"] = torch.zeros(N * per, P, case["heads"], device=dev)
    else:
        s["codes"] = codes(N * per, P, d)
        s["scales"] = normal(N * per, P, case["heads"]).abs() * 0.01 + 1e-4
        s["out"] = torch.empty(total, d, dtype=DTYPES[case["dtype"]], device=dev)
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    do = case["do"]
    if not own:
        return {"lookup": _plain_lookup, "table_grad": _plain_table_grad, "join8": _plain_join8, "cache_write": _plain_write,
                "cache_read": _plain_read, "attend": _plain_attend}[do](s)
    import paper_2108_02191_b200 as robe
    if do == "lookup":
        robe.robe_table_forward(s["table"], s["ids"], s["out"], case["scale"])
        return s["out"]
    if do == "table_grad":
        robe.robe_table_backward(s["grad"], s["ids"], s["grad_table"], s["workspace"], case["scale"], case["accumulate"])
        return s["grad_table"]
    if do == "join8":
        norm = robe.ROBE_NORM_RMS if case["norm"] == "rms" else robe.ROBE_NORM_LAYER
        robe.robe_residual_quantize(s["x"], s["residual"], s["out"], s["codes"], s["scales"], s["w"], case["group"], case["scale"], norm, EPS)
        return [s["out"], s["codes"], s["scales"]]
    if do == "cache_write":
        robe.robe_cache_write(s["rows"], s["codes"], s["scales"], s["pages"], s["offsets"], s["starts"], case["dim"])
        return [s["codes"], s["scales"]]
    if do == "attend":
        robe.robe_cache_attention(s["q"], s["keys"], s["keys_scales"], s["values"], s["values_scales"], s["pages"], s["starts"], s["out"],
                                  s["workspace"], 1.0 / math.sqrt(case["dim"]), s["bias"], s["bias_rows"])
        return s["out"]
    robe.robe_cache_read(s["codes"], s["scales"], s["pages"], s["out"], s["offsets"], s["starts"], case["dim"])
    return s["out"]


# ---- plain forms


def _plain_lookup(s):
    return (s["table"][s["ids"].long()].float() * s["case"]["scale"]).to(DTYPES[s["case"]["rows"]])


def _plain_table_grad(s):
    g = torch.zeros(s["grad_table"].shape, dtype=torch.float64, device="cuda")
    g.index_add_(0, s["ids"].long(), s["grad"].double())
    g.mul_(s["case"]["scale"])
    if s["case"]["accumulate"]:
        g.add_(s["grad_table"])
    s["grad_table"].copy_(g)
    return s["grad_table"]


def _groups(v, group):
    """[rows, groups, columns of a group], the last group filled up with zeros."""
    rows, d = v.shape
    group = group or d
    short = -d % group
    if short:
        v = torch.cat([v, v.new_zeros(rows, short)], 1)
    return v.reshape(rows, -1, group)


def _quantize(v, group, code):
    """(codes as the type that holds them, scales)"""
    rows, d = v.shape
    v = _groups(v, group)
    scales = v.abs().amax(2).clamp(min=SMALLEST) / LARGEST[code]
    v = (v * (1.0 / scales)[:, :, None]).clamp(-LARGEST[code], LARGEST[code])
    v = v.round() if code == "i8" else v
    return v.to(CODES[code]).reshape(rows, -1)[:, :d], scales


def _plain_join8(s):
    case = s["case"]
    v = s["x"].float() * case["scale"]
    if s["residual"] is not None:
        v = s["residual"].float() + v
    out = v.to(s["x"].dtype)
    if case["norm"] == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * s["w"]
    codes, scales = _quantize(v, case["group"], "e4m3")
    return [out, codes.contiguous(), scales]


def _slots(s):
    """Row of the cache that every row of the batch has its place in."""
    total, P = int(s["offsets"][-1]), s["case"]["page"]
    r = torch.arange(total, device="cuda")
    seq = torch.bucketize(r, s["offsets"][1:], right=True)
    pos = s["starts"][seq] + r - s["offsets"][seq]
    return s["pages"][seq, pos // P].long() * P + pos % P


def _plain_write(s):
    case = s["case"]
    codes, scales = _quantize(s["rows"].float(), case["dim"], case["code"])
    slots = _slots(s)
    d = case["heads"] * case["dim"]
    s["codes"].view(torch.uint8).reshape(-1, d)[slots] = codes.contiguous().view(torch.uint8)
    s["scales"].reshape(-1, case["heads"])[slots] = scales
    return [s["codes"], s["scales"]]


def _plain_read(s):
    case = s["case"]
    slots = _slots(s)
    d = case["heads"] * case["dim"]
    v = s["codes"].view(torch.uint8).reshape(-1, d)[slots].view(CODES[case["code"]]).float()
    v = v.reshape(-1, case["heads"], case["dim"]) * s["scales"].reshape(-1, case["heads"])[slots][:, :, None]
    return v.reshape(-1, d).to(DTYPES[case["dtype"]])


def _edges(case):
    """Smallest distance of every bucket: the first half exact, then equal steps of the logarithm up to `far`."""
    half = case["buckets"] // 2
    steps = case["buckets"] - half
    edges = list(range(half))
    for k in range(steps):
        n = max(half, int(half * (case["far"] / half) ** (k / steps)) - 2)
        while n ** steps < half ** (steps - k) * case["far"] ** k:
            n += 1
        edges.append(n)
    return edges


def _plain_attend(s):
    case = s["case"]
    N, H, G, D = case["N"], case["heads"], case["group"], case["dim"]

    def rows(what):  # [N, H, positions, D], by whole pages
        v = s[what].view(torch.uint8)[s["pages"].long()].view(CODES[case["code"]]).float().reshape(N, -1, H, D)
        return (v * s[what + "_scales"][s["pages"].long()].reshape(N, -1, H, 1)).permute(0, 2, 1, 3)

    q = s["q"].float().reshape(N, H, G, D) / math.sqrt(D)
    scores = q @ rows("keys").transpose(2, 3)
    back = s["starts"][:, None] - torch.arange(scores.shape[3], device="cuda")  # how far behind the new token
    if case["buckets"]:
        bucket = torch.bucketize(back.clamp(min=0), torch.tensor(_edges(case)[1:], device="cuda"), right=True)
        scores = scores + s["bias_rows"][bucket].permute(0, 2, 1).reshape(N, H, G, -1)
    scores = torch.where(back[:, None, None, :] < 0, -math.inf, scores)
    p = torch.exp(scores - scores.amax(3, keepdim=True))
    out = (p / p.sum(3, keepdim=True)) @ rows("values")
    return out.reshape(N, H * G, D).to(torch.bfloat16)


# ---------------------------------------------------------------- 64 bits, from the definitions


def exact(case, seed):
    s = prepare(case, seed)
    return {"lookup": _exact_lookup, "table_grad": _exact_table_grad, "join8": _exact_join8, "cache_write": _exact_write,
            "cache_read": _exact_read, "attend": _exact_attend}[case["do"]](s)


def _exact_lookup(s):
    return torch.index_select(s["table"], 0, s["ids"].to(torch.int64)).to(torch.float64) * s["case"]["scale"]


def _exact_table_grad(s):
    """Sums of runs of equal ids: differences of the running sum over the sorted rows, a block of columns at a time."""
    case = s["case"]
    order = torch.argsort(s["ids"].long(), stable=True)
    present, counts = torch.unique_consecutive(s["ids"].long()[order], return_counts=True)
    ends = counts.cumsum(0)
    total = s["grad_table"].double() if case["accumulate"] else torch.zeros(s["grad_table"].shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // case["n"])
    for c in range(0, case["d"], step):
        upto = s["grad"][:, c:c + step][order].double().cumsum(0)[ends - 1]
        upto[1:] = upto[1:] - upto[:-1].clone()
        total[present, c:c + step] += upto * case["scale"]
    return total


def _exact_codes(v, group, code):
    """(what the codes stand for before they are rounded, scales); v in 64 bits"""
    d = v.shape[1]
    parts = torch.split(v, group or d, 1)
    scales = torch.stack([torch.clamp(p.abs().max(1).values, min=SMALLEST) / LARGEST[code] for p in parts], 1)
    return torch.cat([p / scales[:, k:k + 1] for k, p in enumerate(parts)], 1), scales


def _exact_join8(s):
    case = s["case"]
    out = case["scale"] * s["x"].double()
    if case["residual"]:
        out = out + s["residual"].double()
    centred = out - out.mean(1, keepdim=True) if case["norm"] == "layer" else out
    normed = centred * (centred.square().sum(1, keepdim=True) / case["d"] + EPS).rsqrt() * s["w"].double()
    return [out, *_exact_codes(normed, case["group"], "e4m3")]


def _places(s):
    """(sequence, page's number, row in the page) of every row of the batch, on the host sequence by sequence."""
    P = s["case"]["page"]
    offsets, starts = s["offsets"].tolist(), s["starts"].tolist()
    page, row = [], []
    for n in range(s["case"]["N"]):
        at = torch.arange(starts[n], starts[n] + offsets[n + 1] - offsets[n])
        page.append(s["pages"][n].cpu()[at // P])
        row.append(at % P)
    return torch.cat(page).long().cuda(), torch.cat(row).cuda()


def _exact_write(s):
    case = s["case"]
    codes, scales = _exact_codes(s["rows"].double(), case["dim"], case["code"])
    page, row = _places(s)
    full = torch.zeros(s["scales"].shape, dtype=torch.float64, device="cuda")
    full[page, row] = scales
    if case["code"] == "i8":
        return [None, full]  # (whole numbers: a value between two of them has no exact one)
    values = torch.zeros(s["codes"].shape, dtype=torch.float64, device="cuda")
    values[page, row] = codes
    return [values, full]


def _exact_read(s):
    case = s["case"]
    page, row = _places(s)
    codes = s["codes"].view(torch.uint8)[page, row]
    if case["code"] == "i8":
        v = codes.view(torch.int8).double()
    else:  # sign, four bits of exponent, three of fraction; exponent 0 has no leading one
        c = codes.long()
        e, f = (c >> 3) & 15, (c & 7).double()
        v = torch.where(e > 0, (8 + f) * torch.exp2((e - 10).double()), f * 2.0 ** -9) * torch.where(c > 127, -1.0, 1.0)
    v = v.reshape(-1, case["heads"], case["dim"]) * s["scales"][page, row].double()[:, :, None]
    return v.reshape(-1, case["heads"] * case["dim"])


def _exact_attend(s):
    """Sequence by sequence, head by head."""
    case = s["case"]
    H, G, D, P = case["heads"], case["group"], case["dim"], case["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    half = case["buckets"] // 2
    steps = case["buckets"] - half
    reached = [half ** (steps - k) * case["far"] ** k for k in range(steps)]  # distance ** steps has to reach these
    for n, last in enumerate(s["starts"].tolist()):
        at = torch.arange(last + 1, device="cuda")
        page, row = s["pages"][n].long()[at // P], at % P
        if case["buckets"]:
            near = [b if b < half else half + sum(b ** steps >= r for r in reached) - 1 for b in range(min(last + 1, case["far"]))]
            bucket = torch.full((last + 1,), case["buckets"] - 1)
            bucket[:len(near)] = torch.tensor(near)
            bias = s["bias_rows"].double()[bucket.flip(0).cuda()]
        for h in range(H):
            kv = [s[w].reshape(-1, P, H, D)[page, row, h].double() * s[w + "_scales"][page, row, h].double()[:, None]
                  if case["code"] == "i8" else
                  s[w].view(torch.uint8).reshape(-1, P, H, D)[page, row, h].view(torch.float8_e4m3fn).double()
                  * s[w + "_scales"][page, row, h].double()[:, None] for w in ("keys", "values")]
            scores = kv[0] @ s["q"][n, h * G:(h + 1) * G].double().t() * D ** -0.5
            if case["buckets"]:
                scores = scores + bias[:, h * G:(h + 1) * G]
            out[n, h * G:(h + 1) * G] = torch.softmax(scores, 0).t() @ kv[1]
    return out
