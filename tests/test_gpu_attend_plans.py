"""How attention over a cache cuts its sequences into spans: spans longer than the shortest, several for a CTA, as many as the workspace
has room for, lengths around every span's end, calls of sequences by the lane, by the warp and beyond, and starts past the page table.
The values tell which keys were taken: a column adds up the keys of some steps of 128, or the first or the last of some."""
import math

import pytest
import torch

import paper_2108_02191_b200 as robe
import rows8_reference as ref
import rowops_reference as rowref
from test_gpu_row_ops import NAN, Workspace, gen

KINDS = [torch.float8_e4m3fn, torch.int8]
STEP, FAR = 128, 100


def told_values(n, dim, seed):
    """[n, dim], nothing negative: a column of the first half has the keys of every (dim / 2)-th step, one of the third quarter the first of every
    (dim / 4)-th, one of the last quarter the last; the last key is in the last column too."""
    j = torch.arange(n)
    v = torch.zeros(n, dim)
    half, quarter = dim // 2, dim // 4
    v[j, j // STEP % half] = 0.5 + torch.rand(n, generator=gen(seed))
    for at, base in ((0, half), (STEP - 1, half + quarter)):
        some = j[j % STEP == at]
        v[some, base + some // STEP % quarter] = 1.0
    if n:
        v[n - 1, dim - 1] = 16.0
    return v


def distances_bias(rows, start, n, buckets):
    """Bias of keys 0 .. n-1 for a token at `start`; far keys share the last bucket."""
    index = torch.full((n,), buckets - 1)
    for j in range(max(0, min(n, start - FAR + 1)), n):
        index[j] = rowref.bucket(j - start, buckets, FAR, False)
    return rows.double()[index]


def most_off(q, k, v, scale, bias):
    """(result in 64 bits, how far from it the kernel's may be).  The result's own rounding (2^-8) and a weight's to fp16 (2^-11 of it, or 2^-25 of
    the largest contribution); scores in fp32: dim + 8 roundings of terms whose magnitudes add up to sum |q||k|, a few more of the score
    and of what is taken off it, 2^-22 of the exponential; sums: a warp has at most a quarter of the keys and adds sixteen in one instruction, a
    rounding each and one for taking the sum to another maximum, and some for the joins; values read back in fp32."""
    n, dim = k.shape
    scale = float(torch.tensor(scale, dtype=torch.float32))
    q = q.double()
    x = k @ q * scale + (0.0 if bias is None else bias)
    p = torch.softmax(x, 0)
    out, spread = p @ v, p @ v.abs()
    score = (dim + 8) * 2.0 ** -24 * (k.abs() @ q.abs() * abs(scale)).max() + 8 * 2.0 ** -24 * (x.abs().max() + 140.0)
    sums = (n / 32 + 64) * 2.0 ** -23
    small = 2.0 ** -25 * float((p * v.abs().amax(1)).max()) * n
    return out, 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2 * score + 2.0 ** -20 + sums + 2.0 ** -23) * spread * (1 + 2.0 ** -8) + small + 2.0 ** -130


@pytest.mark.parametrize("n", [700, 3000, 50_000])
def test_a_lost_step_or_key_shows(n):
    # planted in the definition: without one step of keys, without one key at a step's end, with a step twice
    dim = 128
    k, v, q = torch.randn(n, dim, generator=gen(1)).double(), told_values(n, dim, 2).double(), torch.randn(dim, generator=gen(3))
    scale = 0.3 / math.sqrt(dim)
    out, most = most_off(q, k, v, scale, None)
    for step in (0, n // STEP // 2, n // STEP - 1):
        at = torch.arange(step * STEP, (step + 1) * STEP)
        keys = torch.arange(n)
        for taken in (keys[(keys < at[0]) | (keys > at[-1])], keys[keys != at[0]], keys[keys != at[-1]], torch.cat([keys, at])):
            wrong = torch.softmax(k[taken] @ q.double() * scale, 0) @ v[taken]
            assert ((wrong - out).abs() > 2 * most).any()
    wrong = torch.softmax(k[:-1] @ q.double() * scale, 0) @ v[:-1]
    assert ((wrong - out).abs() > 2 * most).any()


def check_call(lengths, heads, group, dim, page_rows, kind, buckets, room=0, starts=None, sample=None, seed=1):
    """One call against the definition, on some query heads of every sequence (or of those in `sample`).  starts: where the new tokens stand, at the last
    of their rows unless given; room: positions that the page table has at least."""
    batch, d, total = len(lengths), heads * dim, sum(lengths)
    per = max([1] + [-(-max(n, room) // page_rows) for n in lengths])
    used = [-(-n // page_rows) for n in lengths]
    num = sum(used) + 1
    order = torch.randperm(num, generator=gen(seed)).int()
    pages = torch.full((batch, per), -1, dtype=torch.int32)
    at = 0
    for s, u in enumerate(used):
        pages[s, :u] = order[at:at + u]
        at += u
    pages = pages.cuda()
    offsets = torch.tensor([0] + list(lengths)).cumsum(0).cuda()
    made = {}
    for what in ("keys", "values"):
        codes = torch.zeros(num, page_rows, d, dtype=torch.uint8, device="cuda").view(kind)
        scales = torch.zeros(num, page_rows, heads, device="cuda")
        if what == "keys":
            rows = torch.randn(total, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        else:
            rows = torch.cat([told_values(n, dim, seed + s).repeat(1, heads) for s, n in enumerate(lengths)]).cuda()
            rows *= 1.0 + torch.arange(heads, device="cuda").repeat_interleave(dim)
        robe.robe_cache_write(rows, codes, scales, pages, offsets, None, dim)
        back = torch.empty_like(rows)
        robe.robe_cache_read(codes, scales, pages, back, offsets, None, dim)
        made[what] = (codes, scales, back.reshape(total, heads, dim))
        del rows
    q = torch.randn(batch, heads * group, dim, generator=gen(seed + 5)).bfloat16().cuda()
    bias_rows = (0.3 * torch.randn(buckets, heads * group, generator=gen(seed + 6))).cuda() if buckets else None
    bias = robe.robe_bias_create(buckets, FAR, False) if buckets else None
    starts = [n - 1 for n in lengths] if starts is None else starts
    scale = 0.3 / math.sqrt(dim)
    ws = Workspace(robe.robe_cache_attention_workspace_bytes(batch, heads, heads * group, dim, per * page_rows))
    out = torch.full(q.shape, NAN, dtype=torch.bfloat16, device="cuda")
    robe.robe_cache_attention(q, *made["keys"][:2], *made["values"][:2], pages, torch.tensor(starts, device="cuda"), out, ws.own, scale, bias, bias_rows)
    assert ws.kept_within()
    if bias:
        robe.robe_bias_destroy(bias)
    first = offsets.tolist()
    for s in range(batch) if sample is None else sample:
        n = min(lengths[s], max(0, starts[s] + 1))
        for h in sorted({0, (heads * group) // 2, heads * group - 1}):
            if n == 0:
                assert torch.equal(out[s, h], torch.zeros_like(out[s, h])) and not torch.signbit(out[s, h]).any()
                continue
            k, v = (made[w][2][first[s]:first[s] + n, h // group].double() for w in ("keys", "values"))
            by = distances_bias(bias_rows[:, h].cpu(), starts[s], n, buckets).cuda() if buckets else None
            want, most = most_off(q[s, h], k, v, scale, by)
            off = (out[s, h].double() - want).abs()
            assert (off <= most).all(), (s, h, n, float((off / most).max()))


AROUND = [STEP * k + e for k in range(2, 17) for e in (-1, 0, 1)]  # around the end of every span of up to 2048 keys
LONG = [
    # (heads, group, dim, page_rows, lengths): shares of a CTA of about 500 to 1100 keys, one span of as many
    (16, 1, 128, 64, [3000, 1, 2500, 700, 129, 4000, 0, 640, 1281, 511, 512, 513]),
    (1, 256, 128, 64, [20_000, 511, 512, 513, 7000, 1]),
    (4, 64, 64, 100, [5000, 14_001, 0, 9000, 383, 384, 385]),
    (2, 40, 96, 16, [40_000, 12_345, 257]),
    (8, 17, 32, 16, AROUND + [30_000]),
    # .. of 1536 and more, still one span up to 2048
    (2, 128, 64, 1, [60_001, 7, 9000, 1663, 1664, 1665]),
    (1, 256, 128, 64, AROUND),
    # .. cut into several of more than 1024
    (1, 256, 128, 64, AROUND + [60_000]),
    (1, 64, 256, 7, [400_000, 33_333, 1023, 1024, 1025]),
    # .. into the most that are made for a CTA, which is what the workspace has room for
    (2, 128, 64, 64, [200_000, 131_073, 100_001, 3]),
    (1, 4096, 128, 256, [20_001, 3, 12_289]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,group,dim,page_rows,lengths", LONG, ids=[f"{c[0]}x{c[1]}x{c[2]}-{len(c[4])}-{max(c[4])}" for c in LONG])
def test_spans_of_long_sequences(heads, group, dim, page_rows, lengths, kind, buckets):
    check_call(lengths, heads, group, dim, page_rows, kind, buckets, room=0 if buckets else 1 << 19)


@pytest.mark.gpu
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("batch", [31, 32, 33, 64, 255, 256, 257, 600, 1025])
def test_calls_of_many_sequences(batch, buckets):
    # sequences of none, one, two and three spans in every group of 32
    some = [0, 1, 256, 257, 700, 33, 512, 513, 128, 129, 64]
    lengths = [some[(k * 7 + k // 32) % len(some)] for k in range(batch)]
    check_call(lengths, 2, 2, 64, 16, KINDS[batch % 2], buckets, sample=sorted({*range(0, batch, 1 + batch // 40), *range(max(0, batch - 4), batch)}))


@pytest.mark.gpu
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("length,batch", [(96, 5), (1024, 5), (8192, 5), (320, 300)])
def test_starts_beyond_the_page_table(length, batch, buckets):
    # all positions of the table, whose distances go by where the token stands; no row is written behind the table's last
    beyond = [length - 1, length, length + 5, 10**12, 2**63 - 1]
    check_call([length] * batch, 2, 3, 64, 32, KINDS[1], buckets, starts=[beyond[s % 5] for s in range(batch)], sample=range(10 if batch > 10 else batch))
