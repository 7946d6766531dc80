"""Rows in 8 bits on the GPU: the join whose norm leaves as codes, the paged cache written and read back, and the attention of one new
token over it, against their definitions; and a model's run of them together."""
import math

import pytest
import torch

import paper_2108_02191_b200 as robe
import rowops_reference as rowref
import rows8_reference as ref
from test_gpu_row_ops import NAN, TYPES, Workspace, blank, gen, place, same_bits, surroundings_kept

pytestmark = pytest.mark.gpu

KINDS = [torch.float8_e4m3fn, torch.int8]


def code_bytes(shape, how="plain"):
    """Codes on the GPU: plain, as columns of a wider matrix, or beginning off every boundary.  What stands around is 0x55."""
    left, right = {"plain": (0, 0), "slice": (16, 16), "odd": (3, 2)}[how]
    wide = torch.full((shape[0], left + shape[1] + right), 0x55, dtype=torch.uint8, device="cuda")
    return wide[:, left:left + shape[1]], wide


# ---------------------------------------------------------------- quantised rows and the join

GROUPS = [(1, 1, 1), (1, 8, 0), (3, 64, 32), (5, 100, 32), (2, 100, 0), (33, 128, 128), (7, 1000, 128), (4, 1001, 0), (9, 96, 96), (2, 257, 256),
          (3, 7, 1), (6, 80, 20), (700, 104, 0), (5, 1000, 40), (64, 24, 24), (2, 4096, 128), (3, 4100, 64), (70, 513, 0), (2, 16384, 128), (1, 16400, 0), (2, 40_000, 64), (2, 20_001, 5),
          (4, 505, 64), (5, 961, 0), (2, 4099, 8), (3, 9001, 128), (2, 777, 16), (6, 519, 256),
          (3, 1040, 96), (3, 2056, 64), (5, 1032, 24), (2, 8192, 256), (3, 680, 8), (4, 1280, 160)]


@pytest.mark.parametrize("how", ["plain", "slice", "odd"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,group", GROUPS)
def test_rows_in_8_bits(rows, d, group, dtype, kind, how):
    # no norm, nothing joined: codes and scales are known to the bit
    x = (torch.randn(rows, d, generator=gen(d)) * torch.exp(3 * torch.randn(rows, 1, generator=gen(1)))).to(dtype)
    x[0, d // 2] = 0.0
    codes, around = code_bytes((rows, d), how)
    groups = -(-d // (group or d))
    scales = blank((rows, groups), torch.float32, how)
    robe.robe_residual_quantize(place(x, how), None, None, codes.view(kind), scales, None, group)
    want, want_scales = ref.quantize(x, group, kind)
    assert torch.equal(codes.cpu(), want) and same_bits(scales.cpu(), want_scales) and surroundings_kept(scales)
    if how != "plain":
        left = codes.storage_offset()
        assert (around[:, :left] == 0x55).all() and (around[:, left + d:] == 0x55).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group", [32, 0])
def test_rows_of_zeros_small_numbers_and_what_is_not_a_number(kind, group):
    d = 300
    x = torch.zeros(8, d)
    x[1, 5] = 2.0 ** -120        # below what scales are made for
    x[2, :] = -0.0
    x[3, 7] = NAN
    x[4, 9] = math.inf
    x[5, :] = torch.randn(d, generator=gen(1))
    x[5, 40] = -math.inf
    x[6, :] = 3e38
    x[7, :] = 1.1754944e-38 * torch.arange(d)
    codes, _ = code_bytes((8, d))
    scales = blank((8, -(-d // (group or d))), torch.float32)
    robe.robe_residual_quantize(x.cuda(), None, None, codes.view(kind), scales, None, group)
    want, want_scales = ref.quantize(x, group, kind)
    assert torch.equal(scales.cpu().isnan(), want_scales.isnan()) and torch.equal(scales.cpu().nan_to_num(-1.0), want_scales.nan_to_num(-1.0))
    back = ref.values(codes.cpu(), scales.cpu(), group, kind)
    bad = ref.values(want, want_scales, group, kind).isnan()
    assert torch.equal(back.isnan(), bad) and bad[3, :32].all() and bad[4, :32].all() and not bad[[0, 1, 2, 6, 7]].any()
    assert torch.equal(codes.cpu()[~bad], want[~bad])


def join_tolerance(d):
    """Half steps of fp32 that the statistics and the norm may be off by, relative: a thread adds at most this many squares one after
    the other, then at most 5 + 16 partial sums are joined; the factor is half of that, with seven more operations."""
    return (max(32, 8 * math.ceil(d / 4096)) + 21) / 2 + 10


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,group,how", [(1, 1, 0, "plain"), (3, 64, 32, "plain"), (5, 100, 0, "odd"), (300, 128, 128, "plain"), (7, 1000, 128, "slice"),
                                              (4, 1001, 0, "plain"), (2, 257, 100, "odd"), (2000, 40, 0, "plain"), (3, 4096, 128, "plain"),
                                              (40, 5120, 64, "plain"), (6, 505, 64, "plain"), (5, 961, 0, "odd"), (3, 4099, 8, "plain"), (3, 9001, 128, "slice"), (2, 16384, 128, "plain"), (2, 16400, 0, "slice"), (2, 40_000, 64, "plain")])
def test_join_with_a_norm_in_8_bits(rows, d, group, how, dtype, kind, layer):
    # numbers in steps of 1/64: the sum is exact, so `out` is known to the bit
    x = (torch.randn(rows, d, generator=gen(d)) * 64).round() / 64
    residual = (torch.randn(rows, d, generator=gen(d + 1)) * 64).round() / 64
    x, residual = x.to(dtype), residual.to(dtype)
    w = 1.0 + 0.3 * torch.randn(d, generator=gen(2))
    for res in (residual, None):
        codes, _ = code_bytes((rows, d), how)
        scales = blank((rows, -(-d // (group or d))), torch.float32, how)
        out = blank((rows, d), dtype, how)
        norm = robe.ROBE_NORM_LAYER if layer else robe.ROBE_NORM_RMS
        robe.robe_residual_quantize(place(x, how), place(res, how), out, codes.view(kind), scales, w.cuda(), group, 0.5, norm, 1e-3)
        joined = 0.5 * x.double()
        joined = res.double() + joined if res is not None else joined
        assert same_bits(out.cpu(), joined.to(dtype)) and surroundings_kept(out)
        centred = joined - joined.mean(1, keepdim=True) if layer else joined
        normed = centred / (centred.square().mean(1, keepdim=True) + torch.tensor(1e-3, dtype=torch.float32).double()).sqrt() * w.double()
        near = join_tolerance(d) * 2.0 ** -24
        # a mean is off by its own roundings, which every column then has
        off = near * normed.abs() + (2 * near * joined.abs().mean(1, keepdim=True) / centred.square().mean(1, keepdim=True).add(1e-3).sqrt()
                                     * w.double().abs() if layer else 0.0)
        _, want_scales = ref.quantize(normed.float(), group, kind)
        g = group or d
        most = torch.stack([p.max(1).values for p in (off + 2.0 ** -24 * normed.abs()).split(g, 1)], 1)
        q = ref.LARGEST[kind]
        assert ((scales.cpu().double() - want_scales.double()).abs() <= most / q + 2.0 ** -23 * want_scales.double()).all()
        back = ref.values(codes.cpu(), scales.cpu(), group, kind)
        step = scales.cpu().double().repeat_interleave(g, 1)[:, :d]
        # half a step of the code: of whole numbers, or 2^-4 of the value (below 2^-6 half of 2^-9); and two roundings of the quotient
        half = 0.5 * step if kind == torch.int8 else torch.maximum(2.0 ** -4 * normed.abs(), 2.0 ** -10 * step)
        assert ((back - normed).abs() <= half * (1 + 2.0 ** -20) + 2 * off + 2.0 ** -22 * normed.abs()).all()


@pytest.mark.parametrize("rows,d", [(50, 128), (3, 4096), (2, 20_000), (40, 1001), (9, 4099)])
def test_join_in_place(rows, d):
    x, residual, w = torch.randn(rows, d, generator=gen(1)).cuda(), torch.randn(rows, d, generator=gen(2)).cuda(), torch.ones(d, device="cuda")
    def call(residual, out):
        codes, _ = code_bytes((rows, d))
        scales = blank((rows, 1), torch.float32)
        robe.robe_residual_quantize(x, residual, out, codes.view(torch.int8), scales, w, 0)
        return codes, scales
    out = torch.empty_like(x)
    a = call(residual, out)
    b = call(residual, residual)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(out, residual)


def test_join_gradient_is_the_residual_joins():
    # the gradient through the norm: that of differences of the sum over normed (before its rounding to codes) in 64 bits
    rows, d, eps = 4, 24, 1e-3
    x, residual = torch.randn(rows, d, generator=gen(1)), torch.randn(rows, d, generator=gen(2))
    w, go, gn = 1 + 0.2 * torch.randn(d, generator=gen(3)), torch.randn(rows, d, generator=gen(4)), torch.randn(rows, d, generator=gen(5))
    out = torch.empty(rows, d, device="cuda")
    codes, _ = code_bytes((rows, d))
    scales = torch.empty(rows, 1, device="cuda")
    robe.robe_residual_quantize(x.cuda(), residual.cuda(), out, codes.view(KINDS[0]), scales, w.cuda(), 0, 0.5, robe.ROBE_NORM_RMS, eps)
    gx, gr, gw = torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    robe.robe_residual_backward(go.cuda(), gn.cuda(), x.cuda(), out, gx, gr, None, w.cuda(), None, None, gw, None, ws, 0.5, robe.ROBE_NORM_RMS, eps)

    def loss(x, residual, w):
        o = residual + 0.5 * x
        return float((o * go.double()).sum() + (o / (o.square().mean(1, keepdim=True) + eps).sqrt() * w * gn.double()).sum())

    at = [x.double(), residual.double(), w.double()]
    for k, got in enumerate((gx, gr, gw)):
        flat = at[k].reshape(-1)
        for i in range(0, flat.numel(), 7):
            h, keep = 1e-5, float(flat[i])
            flat[i] = keep + h
            up = loss(*at)
            flat[i] = keep - h
            down = loss(*at)
            flat[i] = keep
            # differences: h^2 times third derivatives, and 2^-53 of the sum over h; the kernel's: a few dozen half steps of terms near 1
            assert abs((up - down) / (2 * h) - float(got.reshape(-1)[i])) < 2e-5


def test_rows_of_nothing():
    e = torch.empty(0, 8, device="cuda")
    robe.robe_residual_quantize(e, None, e, e.to(torch.int8), torch.empty(0, 1, device="cuda"), None)


# ---------------------------------------------------------------- the cache


class Cache:
    """Codes [pages, page_rows, d] and scales on the GPU: laid end to end, keys and values of a page behind one another ("pair"), or off
    every boundary ("odd").  Everything starts as 0x55."""

    def __init__(self, pages, page_rows, d, group, kind, how="plain"):
        groups = -(-d // (group or d))
        if how == "pair":
            self.all = torch.full((pages, 2, page_rows, d), 0x55, dtype=torch.uint8, device="cuda")
            self.bytes = self.all[:, 1]
            self.all_scales = torch.full((pages, 2, page_rows, groups), 5.0, device="cuda")
            self.scales = self.all_scales[:, 1]
        else:
            left = 3 if how == "odd" else 0
            self.all = torch.full((pages, page_rows, left + d + 2 * left), 0x55, dtype=torch.uint8, device="cuda")
            self.bytes = self.all[:, :, left:left + d]
            self.all_scales = torch.full((pages, page_rows, groups + left), 5.0, device="cuda")
            self.scales = self.all_scales[:, :, :groups]
        self.codes = self.bytes.view(kind)
        self.kind, self.group, self.d = kind, group, d


def sequences(lengths, page_rows, starts, seed, spare=2):
    """(pages [batch, most] shuffled, number of pages, offsets)"""
    most = max([1] + [-(-(s + n) // page_rows) for s, n in zip(starts, lengths)])
    num = len(lengths) * most + spare
    pages = torch.randperm(num, generator=gen(seed))[:len(lengths) * most].reshape(len(lengths), most).int()
    return pages, num, torch.tensor([0] + lengths).cumsum(0)


CASES = [([1], [0], 1, 8, 8), ([1, 1, 1], [5, 0, 17], 4, 64, 32), ([7, 0, 130, 1], [0, 3, 60, 9], 16, 256, 64), ([40, 3], [0, 1], 3, 100, 32),
         ([65, 64, 63], [1, 0, 2], 64, 160, 80), ([5, 6], [0, 0], 5, 1001, 0), ([30], [2], 16, 192, 96), ([9, 9], [7, 8], 8, 1024, 128), ([3, 4], [0, 0], 2, 20, 1),
         ([300, 200], [0, 0], 32, 512, 256), ([12], [0], 16, 300, 0), ([3000, 0, 2500], [5, 1, 0], 64, 128, 64), ([2000], [0], 16, 1024, 128),
         ([3000, 0, 2500, 700], [5, 1, 0, 70], 64, 512, 128), ([6200], [0], 16, 512, 8), ([2500], [3], 32, 960, 96), ([5000], [0], 64, 520, 64), ([5000], [9], 64, 512, 16)]


@pytest.mark.parametrize("how", ["plain", "pair", "odd"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,starts,page_rows,d,group", CASES)
def test_cache_write_and_read(lengths, starts, page_rows, d, group, dtype, kind, how):
    pages, num, offsets = sequences(lengths, page_rows, starts, d)
    n = int(offsets[-1])
    rows = torch.randn(n + 3, d, generator=gen(n)).to(dtype)  # three rows behind the last sequence
    rows[:, ::7] *= 30
    cache = Cache(num, page_rows, d, group, kind, how)
    want, want_scales = cache.all.cpu().clone(), cache.all_scales.cpu().clone()
    rows_at = "odd" if how == "odd" else "plain"
    robe.robe_cache_write(place(rows, rows_at), cache.codes, cache.scales, pages.cuda(), offsets.cuda(), torch.tensor(starts).cuda(), group)
    at = ref.places(pages, page_rows, num, n, offsets.tolist(), starts)
    codes, scales = ref.quantize(rows[:n], group, kind)
    blank_codes, blank_scales = cache.bytes.cpu(), cache.scales.cpu()
    if how == "pair":
        view, view_scales = want[:, 1], want_scales[:, 1]
    else:
        left = 3 if how == "odd" else 0
        view, view_scales = want[:, :, left:left + d], want_scales[:, :, :scales.shape[1]]
    for r, p in enumerate(at):
        view[p // page_rows, p % page_rows] = codes[r]
        view_scales[p // page_rows, p % page_rows] = scales[r]
    assert torch.equal(cache.all.cpu(), want) and torch.equal(cache.all_scales.cpu(), want_scales)
    assert blank_codes.shape == view.shape and blank_scales.shape == view_scales.shape
    # and back
    out = blank((n + 3, d), dtype, rows_at)
    robe.robe_cache_read(cache.codes, cache.scales, pages.cuda(), out, offsets.cuda(), torch.tensor(starts).cuda(), group)
    back = ref.values(codes, scales, group, kind)  # (code * scale has at most 31 bits: exact in 64, once rounded in fp32)
    assert same_bits(out.cpu()[:n], back.float().to(dtype)) and out[n:].isnan().all() and surroundings_kept(out)
    # what was written is within half a step
    step = scales.double().repeat_interleave(group or d, 1)[:, :d]
    half = 0.5 * step if kind == torch.int8 else torch.maximum(2.0 ** -4 * rows[:n].double().abs(), 2.0 ** -10 * step)
    assert ((back - rows[:n].double()).abs() <= half * (1 + 2.0 ** -20) + 2.0 ** -22 * rows[:n].double().abs()).all()


@pytest.mark.parametrize("group", [32, 0])
@pytest.mark.parametrize("equal", [False, True])
def test_cache_rows_without_a_place(group, equal):
    page_rows, num, d = 4, 6, 320
    pages = torch.tensor([[0, -1, 5], [6, 2, 2**31 - 1], [3, 4, -2**31]], dtype=torch.int32)
    starts = [-3, 2, 2**62]
    lengths = [9, 9, 9] if equal else [9, 13, 4]
    offsets = torch.tensor([0] + lengths).cumsum(0) + (0 if equal else 2)
    n = int(offsets[-1]) + (0 if equal else 1)
    rows = torch.randn(n, d, generator=gen(1))
    cache = Cache(num, page_rows, d, group, torch.int8)
    want, want_scales = cache.bytes.cpu().clone(), cache.scales.cpu().clone()
    at = ref.places(pages, page_rows, num, n, offsets.tolist(), starts)
    offs = None if equal else offsets.cuda()
    robe.robe_cache_write(rows.cuda(), cache.codes, cache.scales, pages.cuda(), offs, torch.tensor(starts).cuda(), group)
    codes, scales = ref.quantize(rows, group, torch.int8)
    for r, p in enumerate(at):
        if p >= 0:
            want[p // page_rows, p % page_rows], want_scales[p // page_rows, p % page_rows] = codes[r], scales[r]
    assert torch.equal(cache.bytes.cpu(), want) and torch.equal(cache.scales.cpu(), want_scales)
    out = blank((n, d), torch.float32)
    robe.robe_cache_read(cache.codes, cache.scales, pages.cuda(), out, offs, torch.tensor(starts).cuda(), group)
    back = ref.values(codes, scales, group, torch.int8).float()
    for r, p in enumerate(at):
        if p == -2:
            assert out[r].isnan().all()
        elif p == -1:
            assert torch.equal(out[r], torch.zeros_like(out[r])) and not torch.signbit(out[r]).any()
        else:
            assert torch.equal(out[r].cpu(), back[r])
    assert {-1} <= {p for p in at if p < 0} and (equal or -2 in at)


def test_cache_of_many_short_sequences():
    # sequences of no rows between others, several to a block of rows, and a long one among them
    lengths = [k * k % 4 * (k % 3) for k in range(1500)] + [700] + [0] * 500 + [1] * 40
    pages, num, offsets = sequences(lengths, 4, [k % 5 for k in range(len(lengths))], 3)
    starts = torch.tensor([k % 5 for k in range(len(lengths))])
    n, d = int(offsets[-1]), 64
    rows = torch.randn(n, d, generator=gen(1)).bfloat16()
    cache = Cache(num, 4, d, 32, torch.int8)
    robe.robe_cache_write(rows.cuda(), cache.codes, cache.scales, pages.cuda(), offsets.cuda(), starts.cuda(), 32)
    at = torch.tensor(ref.places(pages, 4, num, n, offsets.tolist(), starts.tolist()))
    codes, scales = ref.quantize(rows, 32, torch.int8)
    assert torch.equal(cache.bytes.cpu().reshape(-1, d)[at], codes) and torch.equal(cache.scales.cpu().reshape(-1, 2)[at], scales)
    out = blank((n, d), torch.float32)
    robe.robe_cache_read(cache.codes, cache.scales, pages.cuda(), out, offsets.cuda(), starts.cuda(), 32)
    assert torch.equal(out.cpu(), ref.values(codes, scales, 32, torch.int8).float())


def test_cache_of_nothing():
    pages = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    cache = Cache(1, 4, 32, 32, KINDS[0])
    rows = torch.randn(4, 32, generator=gen(1)).cuda()
    robe.robe_cache_write(rows[:0], cache.codes, cache.scales, pages, None, None, 32)
    robe.robe_cache_write(rows, cache.codes[:0], cache.scales[:0], pages, None, None, 32)  # no pages at all
    out = torch.full((4, 32), NAN, device="cuda")
    robe.robe_cache_read(cache.codes[:0], cache.scales[:0], pages, out, None, None, 32)
    assert not out.any() and (cache.all == 0x55).all()
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    out.fill_(NAN)
    robe.robe_cache_read(cache.codes, cache.scales, none, out, torch.zeros(1, dtype=torch.int64, device="cuda"), None, 32)
    assert out.isnan().all()  # no sequences: no row is of one


def test_cache_past_2_to_32_bytes():
    # places beyond 32 bits: the last pages of a cache of 4.3 GB
    page_rows, d = 64, 1024
    num = 2**32 // (page_rows * d) + 3
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough memory")
    codes = torch.zeros(num, page_rows, d, dtype=torch.int8, device="cuda")
    scales = torch.zeros(num, page_rows, 8, device="cuda")
    pages = torch.tensor([[num - 1, num - 2], [0, num - 3]], dtype=torch.int32)
    rows = torch.randn(2 * 128, d, generator=gen(1))
    robe.robe_cache_write(rows.cuda(), codes, scales, pages.cuda(), None, None, 128)
    want, want_scales = ref.quantize(rows, 128, torch.int8)
    for s in range(2):
        for k in range(2):
            part = slice(s * 128 + k * 64, s * 128 + (k + 1) * 64)
            assert torch.equal(codes[int(pages[s, k])].view(torch.uint8).cpu(), want[part]) and torch.equal(scales[int(pages[s, k])].cpu(), want_scales[part])
    q = torch.randn(2, 16, 128, generator=gen(2)).bfloat16()
    out = torch.empty_like(q, device="cuda")
    ws = torch.empty(robe.robe_cache_attention_workspace_bytes(2, 8, 16, 128, 128), dtype=torch.uint8, device="cuda")
    robe.robe_cache_attention(q.cuda(), codes, scales, codes, scales, pages.cuda(), torch.tensor([127, 100], device="cuda"), out, ws, 0.1)
    back = ref.values(want, want_scales, 128, torch.int8).reshape(2, 128, 8, 128)
    for s, n in enumerate((128, 101)):
        for h in range(16):
            k = back[s, :n, h // 2]
            attention_close(out[s, h].cpu(), q[s, h], k, k, 0.1, None, torch.int8)


# ---------------------------------------------------------------- attention


def attention_close(got, q, k, v, scale, bias, kind, v_scales=None):
    """One head's result against the definition in 64 bits.  The result's own rounding (2^-8); a weight's to fp16 (2^-11 of it, and
    2^-25 of the largest weight where it is small, for every key); scores in fp32: dim + 8 roundings of terms whose magnitudes add up to
    sum |q||k|, a few more of the score and of what is taken off it, and 2^-22 of the exponential itself."""
    scale = float(torch.tensor(scale, dtype=torch.float32))
    q = q.double()
    out, p = ref.attention(q[None] * scale, k, v, None if bias is None else bias[:, None])
    out, p = out[0], p[0]
    x = k @ q * scale + (0.0 if bias is None else bias)
    grown = (k.abs() @ q.abs() * abs(scale)).max()
    score = (k.shape[1] + 8) * 2.0 ** -24 * grown + 8 * 2.0 ** -24 * (x.abs().max() + 140.0)
    spread = p @ v.abs()
    largest_code = v.abs().amax(1)
    small = 2.0 ** -25 * float((p * largest_code).max()) * k.shape[0]
    most = 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2 * score + 2.0 ** -20) * spread * (1 + 2.0 ** -8) + small + 2.0 ** -130
    assert ((got.double() - out).abs() <= most).all()


def attention_case(lengths, heads, group, dim, page_rows, kind, buckets, seed, room=0, how="plain"):
    """A filled cache of keys and one of values, what they stand for, and queries."""
    batch, d = len(lengths), heads * dim
    pages, num, _ = sequences([max(n, room) for n in lengths], page_rows, [0] * batch, seed)
    made = {}
    for what in ("keys", "values"):
        rows = torch.randn(sum(lengths), d, generator=gen(seed + len(what)))
        rows[:, 1::11] *= 6
        rows *= torch.exp(torch.randn(sum(lengths), 1, generator=gen(seed + 9)))
        cache = Cache(num, page_rows, d, dim, kind, how)
        offsets = torch.tensor([0] + lengths).cumsum(0)
        robe.robe_cache_write(rows.cuda(), cache.codes, cache.scales, pages.cuda(), offsets.cuda(), None, dim)
        codes, scales = ref.quantize(rows, dim, kind)
        made[what] = cache
        made[what + "_rows"] = ref.values(codes, scales, dim, kind).reshape(-1, heads, dim).split(lengths)
    q = torch.randn(batch, heads * group, dim, generator=gen(seed + 5)).bfloat16()
    bias_rows = torch.randn(buckets, heads * group, generator=gen(seed + 6)) if buckets else None
    return made, pages, q, bias_rows


def run_attention(made, pages, q, starts, heads, scale, bias=None, bias_rows=None, room=None):
    page_rows = made["keys"].codes.shape[1]
    ws = Workspace(robe.robe_cache_attention_workspace_bytes(q.shape[0], heads, q.shape[1], q.shape[2], pages.shape[1] * page_rows))
    out = torch.full(q.shape, NAN, dtype=torch.bfloat16, device="cuda")
    robe.robe_cache_attention(q.cuda(), made["keys"].codes, made["keys"].scales, made["values"].codes, made["values"].scales, pages.cuda(),
                              torch.tensor(starts, device="cuda"), out, ws.own, scale, bias, None if bias_rows is None else bias_rows.cuda())
    assert ws.kept_within()
    return out.cpu()


ATTEND = [([1], 1, 1, 32, 1), ([256, 257], 1, 3, 64, 16), ([40] * 300, 1, 2, 32, 8), ([1, 2, 15], 2, 4, 64, 16), ([16, 17, 33, 100], 4, 2, 128, 16), ([70, 300], 1, 8, 96, 64), ([257, 5, 64], 2, 16, 128, 7),
          ([130], 2, 5, 256, 32), ([63, 65], 1, 16, 256, 64), ([500, 1, 129], 3, 12, 64, 128), ([1000], 1, 20, 96, 100), ([2049, 700], 2, 8, 128, 64),
          ([5000], 1, 33, 32, 1), ([3000, 4000], 8, 1, 128, 64)]


@pytest.mark.parametrize("how", ["plain", "pair"])
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths,heads,group,dim,page_rows", ATTEND)
def test_attention(lengths, heads, group, dim, page_rows, kind, buckets, how):
    made, pages, q, bias_rows = attention_case(lengths, heads, group, dim, page_rows, kind, buckets, dim + group, how=how)
    bias = robe.robe_bias_create(buckets, 100, False) if buckets else None
    scale = 0.7 / math.sqrt(dim)
    out = run_attention(made, pages, q, [n - 1 for n in lengths], heads, scale, bias, bias_rows)
    for s, n in enumerate(lengths):
        k, v = made["keys_rows"][s], made["values_rows"][s]
        by = None
        if buckets:
            index = torch.tensor([rowref.bucket(j - (n - 1), buckets, 100, False) for j in range(n)])
            by = bias_rows.double()[index]
        for h in range(heads * group):
            attention_close(out[s, h], q[s, h], k[:, h // group], v[:, h // group], scale, None if by is None else by[:, h], kind)
    if bias:
        robe.robe_bias_destroy(bias)


def test_attention_with_a_two_sided_bias_takes_its_earlier_side():
    lengths, buckets = [77], 32
    made, pages, q, bias_rows = attention_case(lengths, 1, 4, 64, 16, KINDS[0], buckets, 3)
    bias = robe.robe_bias_create(buckets, 50, True)
    out = run_attention(made, pages, q, [76], 1, 0.1, bias, bias_rows)
    by = bias_rows.double()[torch.tensor([rowref.bucket(j - 76, buckets, 50, True) for j in range(77)])]
    for h in range(4):
        attention_close(out[0, h], q[0, h], made["keys_rows"][0][:, 0], made["values_rows"][0][:, 0], 0.1, by[:, h], KINDS[0])
    robe.robe_bias_destroy(bias)


def test_attention_of_short_lengths_in_a_long_table_and_of_no_keys():
    # page tables with room for far more than there is; a sequence without a key, one whose start is beyond the table
    # (two without a key, in fact; starts beyond the table: test_gpu_attend_plans.py)
    lengths = [40, 3, 200, 64]
    made, pages, q, _ = attention_case(lengths, 2, 4, 128, 16, KINDS[0], 0, 11, room=20_000)
    out = run_attention(made, pages, q, [39, -1, 150, -2**63], 2, 0.1)
    assert torch.equal(out[1], torch.zeros_like(out[1])) and torch.equal(out[3], torch.zeros_like(out[3]))
    for s, n in ((0, 40), (2, 151)):
        for h in range(8):
            attention_close(out[s, h], q[s, h], made["keys_rows"][s][:n, h // 4], made["values_rows"][s][:n, h // 4], 0.1, None, KINDS[0])


def mean_close(got, v, kind):
    """Equal weights: value scales here stay above 2^-14, so that a weight is off by 2^-11 of it, and the result by its own rounding."""
    assert float(v.abs().amax(1).min()) / 448 > 2.0 ** -14
    out = v.mean(0)
    assert ((got.double() - out).abs() <= 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2.0 ** -18) * (1 + 2.0 ** -8) * v.abs().mean(0) + 2.0 ** -130).all()


@pytest.mark.parametrize("lengths", [[1, 20, 33, 700], [5000], [40, 0] * 150], ids=["some", "one", "many"])
@pytest.mark.parametrize("open_buckets", [range(0, 1), range(0, 16), range(16, 31), range(31, 32), range(3, 32, 5), range(0)])
def test_attention_with_buckets_masked_by_infinities(lengths, open_buckets):
    # keys whose bias is -inf do not count, wherever they stand; where none counts the result is +0
    heads, group, buckets = 2, 2, 32
    made, pages, q, bias_rows = attention_case(lengths, heads, group, 64, 16, KINDS[0], buckets, 8)
    closed = [b for b in range(buckets) if b not in open_buckets]
    bias_rows[closed] = -math.inf
    bias = robe.robe_bias_create(buckets, 100, False)
    out = run_attention(made, pages, q, [n - 1 for n in lengths], heads, 0.1, bias, bias_rows)
    robe.robe_bias_destroy(bias)
    for s, n in list(enumerate(lengths))[:8]:
        index = torch.tensor([rowref.bucket(j - (n - 1), buckets, 100, False) for j in range(n)], dtype=torch.int64)
        seen = torch.tensor([int(i) in open_buckets for i in index], dtype=torch.bool)
        for h in range(heads * group):
            k, v = made["keys_rows"][s][seen, h // group], made["values_rows"][s][seen, h // group]
            if k.shape[0] == 0:
                assert torch.equal(out[s, h], torch.zeros(64, dtype=torch.bfloat16))
            else:
                attention_close(out[s, h], q[s, h], k, v, 0.1, bias_rows[:, h].double()[index[seen]], KINDS[0])


@pytest.mark.parametrize("length", [7, 40, 900])
@pytest.mark.parametrize("open_buckets", [range(0, 2), range(2, 31), range(31, 32), range(0)])
def test_attention_with_buckets_of_the_lowest_value(length, open_buckets):
    # next to any other bias the type's lowest value is a mask; alone it takes all keys alike
    buckets = 32
    made, pages, q, bias_rows = attention_case([length], 1, 3, 128, 16, KINDS[0], buckets, 4)
    bias_rows[[b for b in range(buckets) if b not in open_buckets]] = torch.finfo(torch.float32).min
    bias = robe.robe_bias_create(buckets, 100, False)
    out = run_attention(made, pages, q, [length - 1], 1, 0.1, bias, bias_rows)
    robe.robe_bias_destroy(bias)
    index = torch.tensor([rowref.bucket(j - (length - 1), buckets, 100, False) for j in range(length)])
    seen = torch.tensor([int(i) in open_buckets for i in index])
    for h in range(3):
        k, v = made["keys_rows"][0][:, 0], made["values_rows"][0][:, 0]
        if seen.any():
            attention_close(out[0, h], q[0, h], k[seen], v[seen], 0.1, bias_rows[:, h].double()[index[seen]], KINDS[0])
        else:
            mean_close(out[0, h], v, KINDS[0])


def test_attention_does_not_read_the_bias_of_positions_without_a_place():
    # the only key of bucket 3 has no page; its bias is no number
    buckets, lengths = 32, [60]
    made, pages, q, bias_rows = attention_case(lengths, 1, 2, 64, 1, KINDS[0], buckets, 5)
    bias_rows[3] = NAN
    pages[0, 60 - 1 - 3] = -1
    bias = robe.robe_bias_create(buckets, 100, False)
    out = run_attention(made, pages, q, [59], 1, 0.1, bias, bias_rows)
    robe.robe_bias_destroy(bias)
    index = torch.tensor([rowref.bucket(j - 59, buckets, 100, False) for j in range(60)])
    seen = index != 3
    assert int((~seen).sum()) == 1
    for h in range(2):
        attention_close(out[0, h], q[0, h], made["keys_rows"][0][seen, 0], made["values_rows"][0][seen, 0], 0.1, bias_rows[:, h].double()[index[seen]], KINDS[0])


@pytest.mark.parametrize("batch", [3, 300])
def test_attention_over_a_cache_without_pages_and_of_no_keys_at_all(batch):
    cache = Cache(2, 16, 64, 64, KINDS[0])
    empty = dict(keys=type(cache).__new__(Cache), values=None)
    empty["keys"].codes, empty["keys"].scales = cache.codes[:0], cache.scales[:0]
    empty["values"] = empty["keys"]
    pages = torch.zeros(batch, 40, dtype=torch.int32)
    q = torch.ones(batch, 4, 64, dtype=torch.bfloat16)
    out = run_attention(empty, pages, q, [600] * batch, 1, 0.1)
    assert torch.equal(out, torch.zeros_like(out))
    out = run_attention(dict(keys=cache, values=cache), pages, q, [-1] * batch, 1, 0.1)
    assert torch.equal(out, torch.zeros_like(out))


def test_attention_leaves_out_positions_without_a_place():
    lengths = [200, 90]
    made, pages, q, _ = attention_case(lengths, 1, 8, 64, 16, KINDS[1], 0, 4)
    bad = pages.clone()
    bad[0, 3], bad[0, 7], bad[1, :] = -1, 2**30, -5
    out = run_attention(made, bad, q, [199, 89], 1, 0.2)
    assert torch.equal(out[1], torch.zeros_like(out[1]))
    keep = [j for j in range(200) if j // 16 not in (3, 7)]
    for h in range(8):
        attention_close(out[0, h], q[0, h], made["keys_rows"][0][keep, 0], made["values_rows"][0][keep, 0], 0.2, None, KINDS[1])
    # a start beyond the table: all positions that the table has
    # (that it runs and leaves the other sequence alone; the values of such a call: test_gpu_attend_plans.py)
    out = run_attention(made, pages, q, [pages.shape[1] * 16 + 10**12, 89], 1, 0.2)
    assert torch.isfinite(out[1].float()).all()


def test_attention_of_large_scores_and_uneven_values():
    # scores of several hundred, far apart; values whose scales span 2^60: what a weight is rounded by goes by contributions
    dim, n = 64, 300
    pages = torch.arange(20, dtype=torch.int32)[None]
    keys, values = torch.randn(n, dim, generator=gen(1)) * 40, torch.randn(n, dim, generator=gen(2))
    values *= torch.exp2(torch.randint(-30, 31, (n, 1), generator=gen(3)).float())
    q = torch.randn(1, 4, dim, generator=gen(4)).bfloat16()
    q[0, 1] = 0.0
    q[0, 2] *= 1e30
    q[0, 3] *= 2.0 ** -120
    made = {}
    for what, rows in (("keys", keys), ("values", values)):
        cache = Cache(20, 16, dim, dim, KINDS[0])
        robe.robe_cache_write(rows.cuda(), cache.codes, cache.scales, pages.cuda(), None, None, dim)
        made[what], made[what + "_rows"] = cache, ref.values(*ref.quantize(rows, dim, KINDS[0]), dim, KINDS[0])
    for h, scale in ((0, 1.0), (1, 1.0), (2, 1e-30), (3, 1.0)):
        out = run_attention(made, pages, q, [n - 1], 1, scale)
        attention_close(out[0, h], q[0, h], made["keys_rows"], made["values_rows"], scale, None, KINDS[0])


def test_attention_of_what_is_not_a_number():
    lengths = [50, 50, 50]
    made, pages, q, _ = attention_case(lengths, 2, 2, 64, 16, KINDS[0], 0, 8)
    # a NaN row behind a sequence's end is not looked at; one inside makes its head NaN and no other
    row = torch.full((1, 128), 1.0)
    row[0, 70] = NAN
    for s, pos in ((0, 50), (1, 20)):
        robe.robe_cache_write(row.cuda(), made["values"].codes, made["values"].scales, pages[s:s + 1].cuda(), None, torch.tensor([pos], device="cuda"), 64)
    out = run_attention(made, pages, q, [49, 49, 49], 2, 0.1)
    assert torch.isfinite(out[0].float()).all() and torch.isfinite(out[2].float()).all()
    assert out[1, 2:].isnan().all() and torch.isfinite(out[1, :2].float()).all()
    q[2, 3, 5] = NAN
    out = run_attention(made, pages, q, [49, 49, 49], 2, 0.1)
    assert out[2, 3].isnan().all() and torch.isfinite(out[2, :3].float()).all()


def test_attention_of_many_sequences():
    batch, dim = 3000, 32
    lengths = [1 + (7 * k) % 23 for k in range(batch)]
    made, pages, q, _ = attention_case(lengths, 1, 2, dim, 8, KINDS[1], 0, 1)
    out = run_attention(made, pages, q, [n - 1 for n in lengths], 1, 0.2)
    for s in range(0, batch, 61):
        for h in range(2):
            attention_close(out[s, h], q[s, h], made["keys_rows"][s][:, 0], made["values_rows"][s][:, 0], 0.2, None, KINDS[1])


def test_attention_bits_and_strides():
    # the same call gives the same bits; queries and results as columns of wider tensors
    lengths = [900, 350]
    made, pages, q, _ = attention_case(lengths, 2, 4, 128, 32, KINDS[0], 0, 2)
    a, b = (run_attention(made, pages, q, [899, 349], 2, 0.1) for _ in range(2))
    assert same_bits(a, b)
    for how in ("slice", "odd"):
        wide_q, out = place(q.reshape(16, 128), how), blank((16, 128), torch.bfloat16, how)
        view = lambda t: t.as_strided((2, 8, 128), (8 * t.stride(0), t.stride(0), 1), t.storage_offset())
        ws = torch.empty(robe.robe_cache_attention_workspace_bytes(2, 2, 8, 128, pages.shape[1] * 32), dtype=torch.uint8, device="cuda")
        robe.robe_cache_attention(view(wide_q), made["keys"].codes, made["keys"].scales, made["values"].codes, made["values"].scales, pages.cuda(),
                                  torch.tensor([899, 349], device="cuda"), view(out), ws, 0.1)
        assert same_bits(out.cpu().reshape(2, 8, 128), a) and surroundings_kept(out)
    # queries in a row with the new keys and values, results in a row of the same length or elsewhere in the queries' own
    for left in (0, 4, 1):
        qkv, wide = torch.randn(2, 12 * 128 + 8, generator=gen(left)).bfloat16().cuda(), torch.full((2, 12 * 128 + 8), NAN, dtype=torch.bfloat16, device="cuda")
        view = lambda t: t[:, left:left + 8 * 128].unflatten(1, (8, 128))
        view(qkv).copy_(q)
        robe.robe_cache_attention(view(qkv), made["keys"].codes, made["keys"].scales, made["values"].codes, made["values"].scales, pages.cuda(),
                                  torch.tensor([899, 349], device="cuda"), view(wide), ws, 0.1)
        assert same_bits(view(wide).cpu(), a) and wide[:, :left].isnan().all() and wide[:, left + 8 * 128:].isnan().all()
    both = torch.randn(2, 2, 8, 128, generator=gen(3)).bfloat16().cuda()
    both[:, 0] = q.cuda()
    robe.robe_cache_attention(both[:, 0], made["keys"].codes, made["keys"].scales, made["values"].codes, made["values"].scales, pages.cuda(),
                              torch.tensor([899, 349], device="cuda"), both[:, 1], ws, 0.1)
    assert same_bits(both[:, 1].cpu(), a) and same_bits(both[:, 0].cpu(), q)


def test_two_captured_attentions_share_a_workspace():
    # other lengths, caches and queries; each replayed after the other, and the second on what the first has left
    calls, want = [], []
    ws = torch.empty(robe.robe_cache_attention_workspace_bytes(3, 2, 8, 64, 60 * 32), dtype=torch.uint8, device="cuda")
    for seed, lengths in ((1, [1900, 3, 700]), (2, [20, 1500, 0])):
        made, pages, q, _ = attention_case(lengths, 2, 4, 64, 32, KINDS[seed - 1], 0, seed, room=1920)
        out = torch.full(q.shape, NAN, dtype=torch.bfloat16, device="cuda")
        args = (q.cuda(), made["keys"].codes, made["keys"].scales, made["values"].codes, made["values"].scales, pages.cuda(),
                torch.tensor(lengths, device="cuda") - 1, out, ws, 0.1)
        calls.append(args)
        want.append(run_attention(made, pages, q, [n - 1 for n in lengths], 2, 0.1))
    graphs = []
    for args in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            robe.robe_cache_attention(*args)
        graphs.append(graph)
    for k in (0, 1, 0, 0, 1, 1, 0):
        calls[k][7].fill_(NAN)
        graphs[k].replay()
        assert same_bits(calls[k][7].cpu(), want[k])


# ---------------------------------------------------------------- together


def test_both_ways_of_calling_give_the_same(monkeypatch):
    lengths = [30, 41]
    made, pages, q, bias_rows = attention_case(lengths, 2, 2, 64, 16, KINDS[0], 16, 2)
    bias = robe.robe_bias_create(16, 40, False)
    x, w = torch.randn(71, 128, generator=gen(3)).bfloat16(), torch.randn(128, generator=gen(4))
    offsets = torch.tensor([0, 30, 71], device="cuda")

    def all_of_them():
        out, codes, scales = torch.empty(71, 128, dtype=torch.bfloat16, device="cuda"), code_bytes((71, 128))[0], torch.empty(71, 4, device="cuda")
        robe.robe_residual_quantize(x.cuda(), x.cuda(), out, codes.view(torch.int8), scales, w.cuda(), 32, 0.5, robe.ROBE_NORM_LAYER)
        cache = Cache(made["keys"].codes.shape[0], 16, 128, 64, torch.int8)
        robe.robe_cache_write(x.cuda(), cache.codes, cache.scales, pages.cuda(), offsets, None, 64)
        back = torch.empty(71, 128, device="cuda")
        robe.robe_cache_read(cache.codes, cache.scales, pages.cuda(), back, offsets, None, 64)
        return [out.float(), codes, scales, cache.all, back, run_attention(made, pages, q, [29, 40], 2, 0.1, bias, bias_rows).float()]

    a = all_of_them()
    native = robe.binding._native
    spare = Cache(made["keys"].codes.shape[0], 16, 128, 64, torch.int8)
    assert native.cache_write(x.cuda(), spare.codes, spare.scales, pages.cuda(), offsets, None, 64, None) == robe.ROBE_OK  # (taken)
    for name in ("residual_quantize", "cache_write", "cache_read", "cache_attention"):
        monkeypatch.setattr(native, name, lambda *_: 1, raising=False)
    b = all_of_them()
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    codes, scales = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 2, device="cuda")
    cache = Cache(3, 4, 64, 32, KINDS[0])
    pages = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    q, starts = torch.zeros(1, 4, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    ws = torch.empty(robe.robe_cache_attention_workspace_bytes(1, 2, 4, 32, 8), dtype=torch.uint8, device="cuda")
    attend = lambda **o: robe.robe_cache_attention(**{**dict(q=q, keys=cache.codes, key_scales=cache.scales, values=cache.codes, value_scales=cache.scales,
                                                             pages=pages, starts=starts, out=torch.empty_like(q), workspace=ws, scale=1.0), **o})
    attend()
    for bad in [lambda: robe.robe_residual_quantize(x, None, None, codes.view(torch.uint8), scales, w, 32),
                lambda: robe.robe_residual_quantize(x, None, None, codes, scales, w, 16), lambda: robe.robe_residual_quantize(x, None, None, codes[:3], scales, w, 32),
                lambda: robe.robe_residual_quantize(x, x.bfloat16(), None, codes, scales, w, 32), lambda: robe.robe_residual_quantize(x, None, None, codes, scales, w[:3], 32),
                lambda: robe.robe_residual_quantize(x, None, None, codes, None, w, 32), lambda: robe.robe_residual_quantize(x.cpu(), None, None, codes, scales, w, 32),
                lambda: robe.robe_cache_write(x, cache.codes, cache.scales, pages.long(), None, None, 32),
                lambda: robe.robe_cache_write(x, cache.codes, cache.scales, pages, starts.int(), None, 32),
                lambda: robe.robe_cache_write(x, cache.codes, cache.scales, pages, starts, None, 32), lambda: robe.robe_cache_write(x, cache.codes, cache.scales[:2], pages, None, None, 32),
                lambda: robe.robe_cache_write(x[:, :32], cache.codes, cache.scales, pages, None, None, 32),
                lambda: robe.robe_cache_read(cache.codes, cache.scales, pages, x.half(), None, None, 32), lambda: robe.robe_cache_read(cache.codes[0], cache.scales, pages, x, None, None, 32),
                lambda: attend(q=q.float()), lambda: attend(q=q[0]), lambda: attend(starts=None), lambda: attend(out=torch.empty_like(q).float()),
                lambda: attend(pages=pages.expand(2, 2)), lambda: attend(values=Cache(3, 4, 64, 32, KINDS[0]).codes[:2]),
                lambda: attend(bias=robe.robe_bias_create(8, 20, False)), lambda: attend(bias=robe.robe_bias_create(8, 20, False), bias_rows=torch.zeros(7, 4, device="cuda"))]:
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad, status in [(lambda: robe.robe_residual_quantize(x, None, None, codes, scales, w, -1), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: robe.robe_residual_quantize(x, None, x, codes, scales, w, 32), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: robe.robe_residual_quantize(x, None, None, codes, scales, w, 32, 1.0, 7), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: robe.robe_residual_quantize(x, None, None, codes, scales, w, 32, 1.0, 0, -1.0), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: robe.robe_cache_write(x, cache.codes, cache.scales, pages.expand(3, 2), None, None, 32), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: attend(values=Cache(3, 4, 64, 32, KINDS[1]).codes), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: attend(values=Cache(3, 4, 64, 32, KINDS[0], "pair").codes), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: attend(keys=Cache(3, 4, 64, 32, KINDS[0], "odd").codes, values=Cache(3, 4, 64, 32, KINDS[0], "odd").codes), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: attend(workspace=None), robe.ROBE_ERR_WORKSPACE), (lambda: attend(workspace=ws[:-300]), robe.ROBE_ERR_WORKSPACE),
                        (lambda: attend(out=q), robe.ROBE_ERR_INVALID_ARG)]:
        with pytest.raises(robe.RobeError) as e:
            bad()
        assert e.value.status == status


def serving_step(s):
    """New tokens of a sequence model: table rows, the join whose norm leaves in 8 bits, keys and values into the cache, attention."""
    robe.robe_table_forward(s["table"], s["ids"], s["x"], 4.0)
    robe.robe_residual_quantize(s["x"], None, s["residual"], s["codes"], s["scales"], s["w"], 64)
    robe.robe_cache_write(s["x"], s["keys"].codes, s["keys"].scales, s["pages"], None, s["starts"], 64)
    robe.robe_cache_write(s["residual"], s["values"].codes, s["values"].scales, s["pages"], None, s["starts"], 64)
    robe.robe_cache_attention(s["x"].view(s["batch"], 4, 64), s["keys"].codes, s["keys"].scales, s["values"].codes, s["values"].scales, s["pages"],
                              s["starts"], s["y"], s["workspace"], 0.125, s["bias"], s["bias_rows"])
    robe.robe_residual_forward(s["y"].view(s["batch"], 256), s["residual"], s["residual"])
    s["starts"].add_(1)


@pytest.mark.parametrize("captured", [False, True])
def test_a_models_tokens_from_table_to_attention(captured):
    batch, d, tokens = 3, 256, 40
    bf = dict(dtype=torch.bfloat16, device="cuda")
    pages = torch.randperm(batch * 3, generator=gen(1)).int().reshape(batch, 3)
    s = dict(batch=batch, table=torch.randn(50, d, generator=gen(2)).bfloat16().cuda(), ids=torch.zeros(batch, dtype=torch.int64, device="cuda"),
             x=torch.empty(batch, d, **bf), residual=torch.empty(batch, d, **bf), codes=torch.empty(batch, d, dtype=torch.float8_e4m3fn, device="cuda"),
             scales=torch.empty(batch, 4, device="cuda"), w=torch.ones(d, device="cuda"), keys=Cache(9, 16, d, 64, KINDS[0]), values=Cache(9, 16, d, 64, KINDS[0]),
             pages=pages.cuda(), starts=torch.zeros(batch, dtype=torch.int64, device="cuda"), y=torch.empty(batch, 4, 64, **bf),
             bias=robe.robe_bias_create(8, 20, False), bias_rows=torch.randn(8, 4, generator=gen(3)).cuda(),
             workspace=torch.empty(robe.robe_cache_attention_workspace_bytes(batch, 4, 4, 64, 48), dtype=torch.uint8, device="cuda"))
    history = torch.zeros(batch, 0, d)
    step = lambda: serving_step(s)
    if captured:
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            serving_step(s)
        step = graph.replay
    for t in range(tokens):
        ids = torch.randint(0, 50, (batch,), generator=gen(100 + t))
        s["ids"].copy_(ids)
        step()
        x = s["table"].cpu()[ids].float() * 4.0
        x = x.bfloat16().float()
        history = torch.cat([history, x[:, None]], 1)
        if t % 13 and t + 1 < tokens:
            continue
        rows = ref.values(*ref.quantize(history.reshape(-1, d), 64, KINDS[0]), 64, KINDS[0]).reshape(batch, t + 1, 4, 64)
        index = torch.tensor([rowref.bucket(j - t, 8, 20, False) for j in range(t + 1)])
        for n in range(batch):
            for h in range(4):
                attention_close(s["y"][n, h].cpu(), x[n].reshape(4, 64)[h], rows[n, :, h], rows[n, :, h], 0.125, s["bias_rows"].cpu().double()[index, h], KINDS[0])
        # the residual took the attention's result; one rounding
        want = x.double() + s["y"].cpu().double().reshape(batch, d)
        assert ((s["residual"].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -24 * (x.abs() + 1)).all()
    robe.robe_bias_destroy(s["bias"])


def test_a_models_training_step_with_a_table_beside_the_array():
    # rows of a plain table and rows of the hashed array enter one residual; a join in 8 bits; gradients of both sides
    batch, d, vocab = 200, 64, 90
    table, ids = torch.randn(vocab, d, generator=gen(1)), torch.randint(0, vocab, (batch,), generator=gen(2))
    array = (torch.randn(4096, generator=gen(3)) * 0.1).cuda()
    h = robe.robe_create(4096, 16, d, 1, 5)
    robe.robe_attach_array(h, array)
    other = torch.randint(0, 10**6, (batch,), generator=gen(4)).cuda()
    a, b, out = torch.empty(batch, d, device="cuda"), torch.empty(batch, d, device="cuda"), torch.empty(batch, d, device="cuda")
    codes, scales, w = torch.empty(batch, d, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(batch, 1, device="cuda"), (1 + 0.1 * torch.randn(d, generator=gen(5))).cuda()
    robe.robe_table_forward(table.cuda(), ids.cuda(), a, 2.0)
    robe.robe_forward(h, other, None, batch, b)
    robe.robe_residual_quantize(a, b, out, codes, scales, w, 0, 0.5)
    go, gn = torch.randn(batch, d, generator=gen(6)).cuda(), torch.randn(batch, d, generator=gen(7)).cuda()
    ga, gb, gw, gt = torch.empty(batch, d, device="cuda"), torch.empty(batch, d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(vocab, d, device="cuda")
    garray = torch.zeros(4096, device="cuda")
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(batch, d), dtype=torch.uint8, device="cuda")
    robe.robe_residual_backward(go, gn, a, out, ga, gb, None, w, None, None, gw, None, ws, 0.5)
    ws = torch.empty(robe.robe_table_backward_workspace_bytes(batch, vocab, d), dtype=torch.uint8, device="cuda")
    robe.robe_table_backward(ga, ids.cuda(), gt, ws, 2.0)
    robe.robe_backward(h, gb, other, None, batch, garray, 0.0, None)
    t = table.double().requires_grad_()
    r = b.cpu().double().requires_grad_()
    wd = w.cpu().double().requires_grad_()
    o = r + 0.5 * (2.0 * t[ids])
    n = o / (o.square().mean(1, keepdim=True) + 1e-6).sqrt() * wd
    grads = torch.autograd.grad((o * go.cpu().double()).sum() + (n * gn.cpu().double()).sum(), [t, r, wd])
    back = ref.values(codes.cpu().view(torch.uint8), scales.cpu(), 0, KINDS[0])
    assert ((back - n.detach()).abs() <= torch.maximum(2.0 ** -4 * n.detach().abs(), 2.0 ** -10 * scales.cpu().double()) * 1.001).all()
    # fp32 gradients: a few dozen half steps of terms, whose magnitudes a row's norm bounds
    for got, want in zip((gt, gb, gw), grads):
        assert float((got.cpu().double() - want).abs().max()) <= 2.0 ** -24 * 100 * float(want.abs().max())
    assert float((garray.sum().double().cpu() - gb.double().sum().cpu()).abs()) <= 2.0 ** -24 * batch * d * float(gb.abs().max())
    robe.robe_destroy(h)


def test_calls_on_another_stream():
    stream = torch.cuda.Stream()
    x = torch.randn(500, 256, generator=gen(1)).cuda()
    pages = torch.arange(40, dtype=torch.int32).reshape(1, 40).cuda()
    cache, back = Cache(40, 16, 256, 64, torch.int8), torch.empty(500, 256, device="cuda")
    codes, scales = code_bytes((500, 256))[0], torch.empty(500, 4, device="cuda")
    torch.cuda.synchronize()
    robe.robe_residual_quantize(x, None, None, codes.view(torch.int8), scales, None, 64, stream=stream)
    robe.robe_cache_write(x, cache.codes, cache.scales, pages, None, None, 64, stream=stream)
    robe.robe_cache_read(cache.codes, cache.scales, pages, back, None, None, 64, stream=stream)
    stream.synchronize()
    want, want_scales = ref.quantize(x.cpu(), 64, torch.int8)
    assert torch.equal(codes.cpu(), want) and torch.equal(scales.cpu(), want_scales)
    assert torch.equal(back.cpu(), ref.values(want, want_scales, 64, torch.int8).float())
