"""The row operators on the GPU against their definitions in 64 bits: types, odd sizes, strides, alignment, masks, single
tokens, other streams, captured graphs, and a model's run of them together with the lookup."""
import math

import pytest
import torch

import paper_2108_02191_b200 as robe
import rowops_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
NAN = float("nan")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def place(t, how="plain"):
    """A host tensor on the GPU: plain, as columns of a wider matrix, or beginning inside a 16-byte piece.  What stands
    around it is NaN."""
    if t is None:
        return None
    if how == "plain":
        return t.cuda()
    rows = t.reshape(-1, t.shape[-1])
    left, right = {"slice": (16, 16), "odd": (3, 2)}[how]
    wide = torch.full((rows.shape[0], left + rows.shape[1] + right), NAN, dtype=t.dtype, device="cuda")
    wide[:, left:left + rows.shape[1]] = rows.cuda()
    return wide[:, left:left + rows.shape[1]]


def blank(shape, dtype, how="plain"):
    return place(torch.full(shape, NAN, dtype=dtype), how)


def surroundings_kept(t):
    """What stands beside a placed tensor's columns is still NaN."""
    base = t._base
    if base is None:
        return True
    left = t.storage_offset()
    return bool(base[:, :left].isnan().all()) and bool(base[:, left + t.shape[-1]:].isnan().all())


def same_bits(a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


class Workspace:
    """A workspace of the size asked for, full of old bytes, with others behind it that must stay."""

    def __init__(self, size):
        self.all = torch.full((size + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
        self.size = size
        self.own = self.all[:size]

    def kept_within(self):
        return bool((self.all[self.size:] == 0xA5).all())


# ---------------------------------------------------------------- dropout


def dropped(x, p, seed, offset):
    """x (host) dropped: fp32 product with the rounded factor, rounded once."""
    y = (x.float() * torch.tensor(ref.drop_scale(p), dtype=torch.float32)).to(x.dtype)
    return torch.where(ref.kept(x.shape[0], x.shape[1], p, seed, offset), y, torch.zeros((), dtype=x.dtype))


@pytest.mark.parametrize("how", ["plain", "slice", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 9), (64, 16), (33, 100), (200, 128), (17, 213), (2, 4099), (1000, 3),
                                       (1, 70001), (701, 64)])
def test_dropout_matches_the_definition(rows, cols, dtype, how):
    x = torch.randn(rows, cols, generator=gen(rows + cols)).to(dtype)
    p, seed, offset = 0.3, 0x0123456789ABCDEF, (1 << 40) + 5
    out = blank((rows, cols), dtype, how)
    robe.robe_dropout(place(x, how), out, p, seed, offset)
    assert same_bits(out.cpu(), dropped(x, p, seed, offset))
    assert surroundings_kept(out)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.1, 0.5, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1.0])
def test_dropout_probabilities(p):
    x = torch.randn(300, 96, generator=gen(1))
    out = blank((300, 96), torch.float32)
    robe.robe_dropout(x.cuda(), out, p, 11, 3)
    assert same_bits(out.cpu(), dropped(x, p, 11, 3))
    if p == 0.0:
        assert torch.equal(out.cpu(), x)
    if p == 1.0:
        assert not out.any()


@pytest.mark.parametrize("how", ["plain", "odd"])
def test_dropout_in_place_and_of_what_is_not_a_number(how):
    x = torch.randn(40, 72, generator=gen(2)).bfloat16()
    keep = ref.kept(40, 72, 0.5, 5, 9)
    x[~keep] = torch.where(torch.arange(int((~keep).sum())) % 2 == 0, NAN, math.inf).bfloat16()
    t = place(x, how)
    robe.robe_dropout(t, t, 0.5, 5, 9)
    assert torch.isfinite(t).all() and same_bits(t.cpu(), dropped(x, 0.5, 5, 9)) and surroundings_kept(t)


def test_dropout_seeds_and_steps():
    x = torch.ones(64, 64, device="cuda")
    out = torch.empty_like(x)
    for seed, offset, step in [(0, 0, 0), (2**63 + 5, 1, 2), (1, 2**64 - 1, 3), (-1, -1, -1), (7, 3, 2**62)]:
        counter = torch.tensor([step], device="cuda")
        robe.robe_dropout(x, out, 0.5, seed, offset, counter)
        assert torch.equal(out.cpu() != 0, ref.kept(64, 64, 0.5, seed, (offset + step) % 2**64)), (seed, offset, step)


def test_dropout_rows_past_2_to_32_elements():
    # positions beyond 32 bits: the last rows of a matrix of 4.4 G elements
    rows, cols = 1 << 20, 4200
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 9 GB")
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    robe.robe_dropout(x, x, 0.5, 3, 4)
    tail = slice(rows - 64, rows)
    keep = ref.kept(rows, 8, 0.5, 3, 4)[tail]  # (a decision goes by row and column group: the first group is enough)
    assert torch.equal(x[tail, :8].cpu() != 0, keep)
    share = float((x[tail] != 0).float().mean())
    assert abs(share - 0.5) < 5 * 0.5 / math.sqrt(64 * cols)


# ---------------------------------------------------------------- position bias

BUCKETS = [(32, 128, True), (32, 128, False), (6, 20, False), (4, 9, True), (128, 4000, False), (2, 2, False)]


def bias_case(H, q, k, buckets, causal, starts, dtype, seed=0):
    num, far, two_sided = buckets
    rows = torch.randn(num, H, generator=gen(seed))
    index = torch.stack([ref.bias_index(q, k, s, num, far, two_sided, causal) for s in starts])
    return rows, index


SHAPES = [(1, 1, 1, 1, 0), (1, 4, 8, 8, 0), (2, 3, 1, 77, 76), (1, 2, 64, 128, 64), (1, 5, 65, 130, 0), (2, 2, 130, 67, -10),
          (1, 1, 3, 2050, 5), (1, 2, 129, 1025, 900), (3, 1, 40, 40, 1000), (1, 1, 200, 3, -100), (1, 16, 7, 513, 506),
          (1, 1, 1, 1, 2**40), (1, 1, 5, 9, -2**62), (1, 3, 2, 5000, 4998)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H,q,k,start", SHAPES)
def test_bias_forward(N, H, q, k, start, dtype, causal):
    for n, buckets in enumerate(BUCKETS):
        rows, index = bias_case(H, q, k, buckets, causal, [start] * N, dtype, n)
        b = robe.robe_bias_create(*buckets)
        want = torch.where((index < 0)[..., None], -math.inf, rows[index.clamp(min=0)]).permute(0, 3, 1, 2).to(dtype)
        for how in ("plain", "slice", "odd"):
            out = blank((N * H * q, k), dtype, how)
            robe.robe_bias_forward(b, place(rows, how), out.unflatten(0, (N, H, q)), start, causal)
            assert same_bits(out.cpu().reshape(want.shape), want), (buckets, how)
            assert surroundings_kept(out)
        robe.robe_bias_destroy(b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q,k", [(1, 300), (4, 129), (70, 70)])
def test_bias_of_sequences_with_starts_of_their_own(q, k, dtype):
    starts = [k - q, 0, -5, k + 1000, 17, 2**45]
    for causal in (False, True):
        rows, index = bias_case(3, q, k, BUCKETS[0], causal, starts, dtype)
        b = robe.robe_bias_create(*BUCKETS[0])
        want = torch.where((index < 0)[..., None], -math.inf, rows[index.clamp(min=0)]).permute(0, 3, 1, 2).to(dtype)
        out = torch.full((len(starts), 3, q, k), NAN, dtype=dtype, device="cuda")
        robe.robe_bias_forward(b, rows.cuda(), out, torch.tensor(starts, device="cuda"), causal)
        assert same_bits(out.cpu(), want)
        robe.robe_bias_destroy(b)


def bias_grad_reference(g, index, num):
    """(sums, bounds): at most 64 additions in fp32 on a diagonal's way and two where lanes meet, the rest in 64 bits."""
    N, H = g.shape[:2]
    g = g.double()
    want = torch.zeros(num + 1, H, dtype=torch.float64)
    mass = torch.zeros(num + 1, H, dtype=torch.float64)
    for n in range(N):
        of = torch.where(index[n] < 0, num, index[n]).reshape(-1)
        flat = g[n].permute(1, 2, 0).reshape(-1, H)
        want.index_add_(0, of, flat)
        mass.index_add_(0, of, flat.abs())
    return want[:num], 68 * ref.U * mass[:num]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H,q,k,start", SHAPES + [(2, 2, 300, 500, 200), (1, 1, 70, 4500, 4000), (5, 3, 64, 64, 0)])
def test_bias_backward(N, H, q, k, start, dtype, causal):
    for n, buckets in enumerate(BUCKETS):
        _, index = bias_case(H, q, k, buckets, causal, [start] * N, dtype)
        g = torch.randn(N, H, q, k, generator=gen(n)).to(dtype)
        b = robe.robe_bias_create(*buckets)
        want, bound = bias_grad_reference(g, index, buckets[0])
        if causal:  # what stands in masked places has no effect
            g = torch.where((index < 0)[:, None].expand(g.shape), torch.tensor(NAN, dtype=dtype), g)
        bits = None
        for how in ("plain", "slice", "odd"):
            got = blank((buckets[0], H), torch.float32, how)
            ws = Workspace(robe.robe_bias_backward_workspace_bytes(b, H, N, q, k))
            placed = place(g.reshape(N * H * q, k), how).unflatten(0, (N, H, q))
            robe.robe_bias_backward(b, placed, got, ws.own, start, causal)
            assert ws.kept_within()
            ref.assert_within(got, want, bound, (buckets, how))
            assert surroundings_kept(got)
            bits = got.cpu() if bits is None else bits
            assert same_bits(got.cpu(), bits), "alignment changed the result"
        robe.robe_bias_destroy(b)


def test_bias_backward_of_sequences_with_starts_of_their_own():
    starts = [100, 0, -5, 5000, 17, -2**45]
    q, k, H = 33, 141, 3
    for causal in (False, True):
        for dtype in TYPES:
            _, index = bias_case(H, q, k, BUCKETS[0], causal, starts, dtype)
            g = torch.randn(len(starts), H, q, k, generator=gen(4)).to(dtype)
            b = robe.robe_bias_create(*BUCKETS[0])
            want, bound = bias_grad_reference(g, index, 32)
            got = blank((32, H), torch.float32)
            ws = torch.empty(robe.robe_bias_backward_workspace_bytes(b, H, len(starts), q, k), dtype=torch.uint8, device="cuda")
            robe.robe_bias_backward(b, g.cuda(), got, ws, torch.tensor(starts, device="cuda"), causal)
            ref.assert_within(got, want, bound, causal)
            robe.robe_bias_destroy(b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", range(1, 10))
def test_bias_backward_of_few_keys_reads_its_tensor_alone(k, dtype):
    # rows of a few bytes, several of which lie in one 16-byte piece: the pieces of the last matrices' rows end at the tensor's
    # end (on the index-check build a copy that does not is recorded), which is also where its allocation may end
    b = robe.robe_bias_create(*BUCKETS[0])
    size = torch.finfo(dtype).bits // 8
    for N, H, q in [(1, 1, 5), (1, 1, 9), (1, 3, 8), (2, 5, 9), (1, 2, 10), (1, 64, 9), (3, 2, 17), (1, 1, 18), (2, 2, 33), (1, 7, 4)]:
        _, index = bias_case(H, q, k, BUCKETS[0], False, [q // 2 - k] * N, dtype)
        g = torch.randn(N, H, q, k, generator=gen(q)).to(dtype)
        want, bound = bias_grad_reference(g, index, 32)
        ws = Workspace(robe.robe_bias_backward_workspace_bytes(b, H, N, q, k))
        for begin in range(0, 16 // size, 3):  # where the tensor begins in a piece; what stands around it is NaN
            around = torch.full((begin + g.numel() + 64,), NAN, dtype=dtype, device="cuda")
            placed = around[begin:begin + g.numel()].view(g.shape)
            placed.copy_(g)
            got = blank((32, H), torch.float32)
            robe.robe_bias_backward(b, placed, got, ws.own, q // 2 - k)
            assert ws.kept_within()
            ref.assert_within(got, want, bound, (N, H, q, begin))
    robe.robe_bias_destroy(b)


def test_bias_of_nothing():
    b = robe.robe_bias_create(32, 128, True)
    rows = torch.randn(32, 4, device="cuda")
    for shape in [(0, 4, 3, 3), (2, 4, 0, 3), (2, 4, 3, 0)]:
        out = torch.empty(shape, device="cuda")
        robe.robe_bias_forward(b, rows, out)
        got = torch.full((32, 4), NAN, device="cuda")
        robe.robe_bias_backward(b, out, got, None)
        assert not got.any() and not got.isnan().any()  # the gradient of nothing is zero
    robe.robe_bias_destroy(b)


def test_bias_gradient_is_the_transpose_of_the_bias():
    # <bias(rows), g> = <rows, grad(g)>: the bias is linear in its rows
    b = robe.robe_bias_create(32, 128, True)
    rows, g = torch.randn(32, 8, generator=gen(1)).cuda(), torch.randn(1, 8, 500, 600, generator=gen(2)).cuda()
    out, got = torch.empty_like(g), torch.empty_like(rows)
    ws = torch.empty(robe.robe_bias_backward_workspace_bytes(b, 8, 1, 500, 600), dtype=torch.uint8, device="cuda")
    robe.robe_bias_forward(b, rows, out, 50)
    robe.robe_bias_backward(b, g, got, ws, 50)
    left, right = (out.double() * g.double()).sum(), (rows.double() * got.double()).sum()
    mass = (out.double() * g.double()).abs().sum()
    assert abs(left - right) <= 70 * ref.U * mass
    robe.robe_bias_destroy(b)


# ---------------------------------------------------------------- residual join


def join_inputs(rows, d, dtype, gate, post, pre, residual, seed):
    r = gen(seed)
    rnd = lambda *s: torch.randn(*s, generator=r)
    t = {"x": rnd(rows, d).to(dtype), "residual": (1.5 * rnd(rows, d) + 0.3).to(dtype) if residual else None,
         "w_post": 1 + 0.2 * rnd(d) if post else None, "w_pre": 1 + 0.2 * rnd(d) if pre else None}
    shape = {"none": None, "row": (rows, 1)}.get(gate, (rows // gate, d) if isinstance(gate, int) else None)
    t["gate"] = rnd(*shape).to(dtype) if shape else None
    return t


def wide(t):
    return None if t is None else t.double()


JOINS = [  # rows, d, gate, post, pre, residual, p
    (1, 1, "none", True, True, True, 0.0), (3, 8, "row", True, True, True, 0.0), (40, 16, 1, True, True, True, 0.1),
    (26, 64, "row", True, True, True, 0.2), (130, 100, 13, True, True, True, 0.1), (70, 128, "row", True, True, False, 0.0),
    (35, 213, "none", True, True, True, 0.1), (60, 213, 20, True, True, True, 0.3), (33, 257, 1, True, False, True, 0.1),
    (9, 512, 3, False, True, True, 0.5), (12, 520, "none", False, True, False, 0.1), (7, 1000, 7, True, True, True, 0.1),
    (20, 1024, 1, True, True, True, 0.1), (5, 2048, "row", True, True, True, 0.0), (6, 4096, 2, True, True, True, 0.1),
    (3, 4097, 1, True, True, True, 0.1), (4, 8192, 4, True, True, True, 0.1), (2, 12_000, "none", True, True, True, 0.1),
    (2, 20_001, 1, True, True, True, 0.1), (3, 40_000, "row", True, True, True, 0.0), (700, 24, 1, True, True, True, 0.1),
    (1500, 40, 750, True, True, True, 0.1), (1201, 12, "none", True, True, True, 0.0), (640, 128, 2, True, True, True, 0.1),
    (5, 3, "none", True, True, True, 0.0), (1400, 96, 1400, True, True, True, 0.0), (64, 36, 32, True, False, True, 1.0),
    (900, 47, "row", True, True, True, 0.1), (6080, 24, 10, True, True, True, 0.1), (12_000, 8, 2, True, True, True, 0.0),
    (3200, 300, 100, True, True, True, 0.1), (1200, 520, 3, True, True, True, 0.1), (300, 909, "none", True, True, True, 0.1),
    (40, 4100, 5, True, True, True, 0.1), (9, 8191, 1, True, True, True, 0.1), (20_000, 5, 1, True, True, True, 0.2),
    (7, 12_288, 1, True, True, True, 0.1), (600, 8200, 3, True, False, True, 0.1), (300, 8208, 150, True, True, True, 0.0),
    (5, 30_000, 5, False, True, False, 0.3), (160, 8193, "row", True, True, True, 0.1)]


@pytest.mark.parametrize("layer", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,gate,post,pre,residual,p", JOINS)
def test_residual_forward(rows, d, gate, post, pre, residual, p, dtype, layer):
    t = join_inputs(rows, d, dtype, gate, post, pre, residual, rows + d)
    factor = ref.kept(rows, d, p, 21, 34).double() * ref.drop_scale(p) if p else torch.ones(1, 1, dtype=torch.float64)
    want = ref.join(*(wide(t[k]) for k in ("x", "residual", "w_post", "w_pre", "gate")), 0.7, layer, 1e-5, factor)
    step = torch.tensor([30], device="cuda")
    for how in ("plain", "slice", "odd"):
        out, normed = blank((rows, d), dtype, how), blank((rows, d), dtype, how) if pre else None
        vec = lambda v: None if v is None else v.cuda()
        robe.robe_residual_forward(place(t["x"], how), place(t["residual"], how), out, normed, vec(t["w_post"]), vec(t["w_pre"]),
                                   place(t["gate"], how), 0.7, layer, 1e-5, p, 21, 4, step)
        ref.assert_within(out, *want[0], (how, "out"))
        assert surroundings_kept(out)
        if pre:
            ref.assert_within(normed, *want[1], (how, "normed"))
            assert surroundings_kept(normed)


@pytest.mark.parametrize("layer", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,gate,post,pre,residual,p", JOINS)
def test_residual_backward(rows, d, gate, post, pre, residual, p, dtype, layer):
    t = join_inputs(rows, d, dtype, gate, post, pre, residual, rows + d)
    factor = ref.kept(rows, d, p, 21, 34).double() * ref.drop_scale(p) if p else torch.ones(rows, d, dtype=torch.float64)
    r = gen(5)
    out = (1.3 * torch.randn(rows, d, generator=r) + 0.2).to(dtype) if pre else None
    go = torch.randn(rows, d, generator=r).to(dtype) if residual or not pre else None
    gn = torch.randn(rows, d, generator=r).to(dtype) if pre else None
    want = ref.join_grad(wide(go), wide(gn), wide(t["x"]), wide(out), wide(t["w_post"]), wide(t["w_pre"]), wide(t["gate"]), 0.7,
                         layer, 1e-5, factor)
    gates = t["gate"].shape[0] if isinstance(gate, int) else 0
    bits = None
    for how in ("plain", "slice", "odd"):
        vec = lambda v: None if v is None else v.cuda()
        got = {"x": blank((rows, d), dtype, how), "residual": blank((rows, d), dtype, how) if residual else None,
               "gate": blank(tuple(t["gate"].shape), dtype, how) if t["gate"] is not None else None,
               "w_post": blank((d,), torch.float32) if post else None, "w_pre": blank((d,), torch.float32) if pre else None}
        ws = Workspace(robe.robe_residual_backward_workspace_bytes(rows, d, gates))
        robe.robe_residual_backward(place(go, how), place(gn, how), place(t["x"], how), place(out, how), got["x"], got["residual"],
                                    vec(t["w_post"]), vec(t["w_pre"]), place(t["gate"], how), got["w_post"], got["w_pre"],
                                    got["gate"], ws.own, 0.7, layer, 1e-5, p, 21, 34)
        assert ws.kept_within()
        for name, v in got.items():
            if v is not None:
                value, bound = want[name]
                ref.assert_within(v, value, bound, (how, name))
                assert name.startswith("w_") or surroundings_kept(v), (how, name)
        if bits is None:  # a second time: the same bits
            again = {k: None if v is None else torch.empty_like(v) for k, v in got.items()}
            robe.robe_residual_backward(place(go, how), place(gn, how), place(t["x"], how), place(out, how), again["x"],
                                        again["residual"], vec(t["w_post"]), vec(t["w_pre"]), place(t["gate"], how),
                                        again["w_post"], again["w_pre"], again["gate"], ws.own, 0.7, layer, 1e-5, p, 21, 34)
            bits = all(v is None or same_bits(v, again[k]) for k, v in got.items())
            assert bits


def whole_numbers(shape, most, seed, dtype=torch.float32):
    """-most .. most without 0, on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = torch.randint(1, most + 1, shape, generator=g, device="cuda")
    return (n * (2 * torch.randint(0, 2, shape, generator=g, device="cuda") - 1)).to(dtype)


def exact_sums(rows, d, gate, dtype, layer, p, how):
    """Rows of +-1 without eps: a norm is the row itself, and with weights after the join of 0 the gradients of weights and gates are
    sums of whole numbers, none of them 0 without dropout: a row that is lost or taken twice shows in every column."""
    assert float((torch.tensor(1.0) / d) * d) == 1.0  # (the kernels multiply by 1 / d)
    if layer:  # as many of either sign in a row
        assert d % 2 == 0
        columns = 1.0 - 2.0 * (torch.arange(d, device="cuda") % 2)
        x, out = (whole_numbers((rows, 1), 1, n) * columns for n in (1, 2))
    else:
        x, out = (whole_numbers((rows, d), 1, n) for n in (1, 2))
    x, out = x.to(dtype), out.to(dtype)
    t, gn = whole_numbers((rows, d), 3, 3, dtype), whole_numbers((rows, d), 3, 4, dtype)
    shape = {"none": None, "row": (rows, 1)}.get(gate, (rows // gate, d) if isinstance(gate, int) else None)
    g = whole_numbers(shape, 2, 5, dtype) if shape else None
    w_post, w_pre = whole_numbers((d,), 2, 6), torch.zeros(d, device="cuda")
    got = {"w_post": blank((d,), torch.float32), "w_pre": blank((d,), torch.float32),
           "gate": blank(shape, dtype, how) if shape else None}
    ws = Workspace(robe.robe_residual_backward_workspace_bytes(rows, d, rows // gate if isinstance(gate, int) else 0))
    robe.robe_residual_backward(place(t, how), place(gn, how), place(x, how), place(out, how), blank((rows, d), dtype, how),
                                blank((rows, d), dtype, how), w_post, w_pre, place(g, how), got["w_post"], got["w_pre"], got["gate"],
                                ws.own, 0.5, layer, 0.0, p, 7, 8)
    assert ws.kept_within()
    assert torch.equal(got["w_pre"].double(), (gn * out).sum(0, dtype=torch.float64))
    s = 0.5 * t.float() * x.float()
    if p:  # (a half is dropped: twice what is kept)
        s = torch.where(ref.kept(rows, d, p, 7, 8).cuda(), ref.drop_scale(p) * s, torch.zeros((), device="cuda"))
    per = gate if isinstance(gate, int) else 1
    of_rows = s if g is None else s * g.float().repeat_interleave(per, 0)
    assert torch.equal(got["w_post"].double(), of_rows.sum(0, dtype=torch.float64))
    if g is not None:
        s = s * w_post
        want = s.sum(1, keepdim=True, dtype=torch.float64) if gate == "row" else s.reshape(-1, per, d).sum(1, dtype=torch.float64)
        assert torch.equal(got["gate"].double(), want.to(dtype).double())


@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,gate,layer,p", [
    (1, 8, 1, 0, 0.0), (20_000, 5, 1, 0, 0.0), (20_001, 5, "none", 0, 0.0), (12_000, 8, 2, 0, 0.0), (120_000, 8, 2, 1, 0.0),
    (6080, 24, 10, 0, 0.0), (1500, 40, 750, 0, 0.0), (1201, 12, "none", 1, 0.0), (31_003, 100, "row", 1, 0.0), (50_000, 128, 1000, 0, 0.0),
    (41_041, 136, 41, 0, 0.0), (7001, 257, "none", 0, 0.0), (9999, 520, 3, 0, 0.0), (2900, 520, 29, 0, 0.5), (3000, 1024, 1500, 0, 0.0),
    (2003, 4096, "none", 1, 0.0), (4097, 264, 17, 0, 0.5), (500, 8200, 250, 0, 0.0), (449, 8200, "row", 0, 0.5), (300, 12_288, 1, 0, 0.0),
    (400, 20_001, 8, 0, 0.0), (297, 30_000, "none", 0, 0.5)])
def test_residual_sums_of_whole_numbers(rows, d, gate, layer, p, dtype, how):
    exact_sums(rows, d, gate, dtype, layer, p, how)


@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,gate", [(480_000, 264, 100), (700_001, 264, "none"), (330_000, 264, 275), (3_700_003, 8, "none"),
                                         (3_700_000, 5, "row"), (2_000_000, 12, 250), (29_700, 8200, 100), (22_500, 8200, 300),
                                         (40_001, 8200, "none")])
def test_residual_sums_of_whole_numbers_in_chunks_cut_by_their_length(rows, d, gate, dtype, how):
    room(12 * rows * d * 4 + (4 << 30) >> 30)
    exact_sums(rows, d, gate, dtype, 0, 0.0, how)


@pytest.mark.parametrize("rows,d,gate", [(50, 128, "none"), (6, 4096, 1), (5, 213, "row"), (2, 20_001, "none")])
def test_residual_in_place(rows, d, gate):
    # the sum over the residual, the residual's gradient over the output's: the same bits as into buffers of their own
    t = {k: place(v) for k, v in join_inputs(rows, d, torch.bfloat16, gate, True, True, True, 9).items()}
    out, normed = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    args = (t["w_post"], t["w_pre"], t["gate"], 0.5, 0, 1e-6, 0.1, 3, 4)
    robe.robe_residual_forward(t["x"], t["residual"], out, normed, *args)
    stream, normed2 = t["residual"].clone(), torch.empty_like(normed)
    robe.robe_residual_forward(t["x"], stream, stream, normed2, *args)
    assert same_bits(stream, out) and same_bits(normed, normed2)
    go, gn = torch.randn_like(out), torch.randn_like(out)
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(rows, d, rows if gate == 1 else 0), dtype=torch.uint8, device="cuda")
    results = []
    for gr in (torch.empty_like(go), go):
        g = [torch.empty_like(out), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
        gg = torch.empty_like(t["gate"]) if t["gate"] is not None else None
        robe.robe_residual_backward(go, gn, t["x"], out, g[0], gr, t["w_post"], t["w_pre"], t["gate"], g[1], g[2], gg, ws, 0.5, 0,
                                    1e-6, 0.1, 3, 4)
        results.append(g + [gr] + ([gg] if gg is not None else []))
    assert all(same_bits(a, b) for a, b in zip(*results))


def test_residual_gate_and_block_output_from_one_projection():
    # x and gate as the halves of one matrix, their gradients too
    both = torch.randn(64, 512, generator=gen(1)).bfloat16().cuda()
    x, gate = both[:, :256], both[:, 256:]
    go = torch.randn(64, 256, generator=gen(2)).bfloat16().cuda()
    grads = torch.full_like(both, NAN)
    w, gw = torch.ones(256, device="cuda"), torch.empty(256, device="cuda")
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(64, 256, 64), dtype=torch.uint8, device="cuda")
    robe.robe_residual_backward(go, None, x, None, grads[:, :256], None, w, None, gate, gw, None, grads[:, 256:], ws)
    want = ref.join_grad(go.cpu().double(), None, x.cpu().double(), None, torch.ones(256, dtype=torch.float64), None,
                         gate.cpu().double(), 1.0, 0, 1e-6, 1.0)
    for name, got in (("x", grads[:, :256]), ("gate", grads[:, 256:]), ("w_post", gw)):
        ref.assert_within(got, *want[name], name)


@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,d,gate", [(40, 64, "row"), (40, 64, 1), (40, 64, 4), (12, 4096, 1), (12, 4096, "row"), (6, 20_001, "row"),
                                         (6, 20_001, 1), (6, 20_001, 3), (4, 30_000, 2)])
def test_residual_backward_of_what_is_not_a_number_where_it_is_dropped(rows, d, gate, post, dtype, how):
    # the block's and the gate's gradients are as if there were zeros; the residual's is what came in
    t = join_inputs(rows, d, dtype, gate, post, False, True, 3)
    keep = ref.kept(rows, d, 0.5, 5, 9)
    go = torch.randn(rows, d, generator=gen(4)).to(dtype)
    results = []
    for fill in (0.0, NAN, math.inf):
        g = torch.where(keep, go, torch.tensor(fill, dtype=dtype))
        gx, gr, gg = blank((rows, d), dtype, how), blank((rows, d), dtype, how), blank(tuple(t["gate"].shape), dtype, how)
        gw = blank((d,), torch.float32) if post else None
        ws = Workspace(robe.robe_residual_backward_workspace_bytes(rows, d, rows // gate if gate != "row" else 0))
        robe.robe_residual_backward(place(g, how), None, place(t["x"], how), None, gx, gr, place(t["w_post"]), None,
                                    place(t["gate"], how), gw, None, gg, ws.own, 0.7, 0, 1e-5, 0.5, 5, 9)
        torch.testing.assert_close(gr.cpu(), g, rtol=0, atol=0, equal_nan=True)  # (a NaN rounded to bf16 has other bits)
        results.append([gx.cpu(), gg.cpu()] + ([gw.cpu()] if post else []))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_residual_of_no_rows():
    for d in (16, 4096):
        e = torch.empty(0, d, device="cuda")
        w = torch.ones(d, device="cuda")
        robe.robe_residual_forward(e, e, e.clone(), e.clone(), w, w)
        g1, g2 = torch.full((d,), NAN, device="cuda"), torch.full((d,), NAN, device="cuda")
        robe.robe_residual_backward(e, e, e, e, e.clone(), e.clone(), w, w, None, g1, g2)
        assert torch.equal(g1, torch.zeros_like(g1)) and torch.equal(g2, torch.zeros_like(g2))


@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
def test_residual_gate_vectors_of_no_rows(dtype, how):
    # sequences of length zero, a gate vector each: the gates' gradients are zero, not what stood there
    e = torch.empty(0, 21, dtype=dtype, device="cuda")
    gate, gg = place(torch.ones(5, 21, dtype=dtype), how), blank((5, 21), dtype, how)
    w, gw = torch.ones(21, device="cuda"), torch.full((21,), NAN, device="cuda")
    robe.robe_residual_forward(e, e, e.clone(), None, w, None, gate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    robe.robe_residual_backward(e, None, e, None, e.clone(), None, w, None, gate, gw, None, gg, stream=side)
    side.synchronize()
    assert same_bits(gg, torch.zeros_like(gg)) and surroundings_kept(gg) and same_bits(gw, torch.zeros_like(gw))


def test_residual_rows_of_zeros_and_of_infinities():
    # eps alone under the root; an infinite element makes its own row NaN and no other
    x = torch.randn(6, 128, generator=gen(3))
    x[1] = 0.0
    x[4, 7] = math.inf
    w = torch.ones(128, device="cuda")
    for layer in (0, 1):
        out, normed = torch.empty(6, 128, device="cuda"), torch.empty(6, 128, device="cuda")
        robe.robe_residual_forward(x.cuda(), None, out, normed, w, w, norm=layer)
        assert not out[1].any() and not normed[1].any()
        assert torch.isfinite(out[[0, 1, 2, 3, 5]]).all() and torch.isfinite(normed[[0, 1, 2, 3, 5]]).all()
        assert out[4, 7].isnan()


def test_dropout_in_the_join_is_that_of_the_dropout_call():
    x = torch.randn(50, 100, generator=gen(8)).cuda()
    for d in (100, 96, 37):
        v = x[:, :d].contiguous()
        a, b = torch.empty_like(v), torch.empty_like(v)
        robe.robe_dropout(v, a, 0.2, 6, 7)
        robe.robe_residual_forward(v, None, b, p=0.2, seed=6, offset=7)
        assert same_bits(a, b)


# ---------------------------------------------------------------- beyond 32 bits


def room(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GB")


def test_residual_of_more_than_2_to_31_elements():
    # the same 1000 rows over and over: the last ones come out as the first
    d, block, times = 4096, 1000, 530
    room(40)
    r = gen(4)
    some = lambda: torch.randn(block, d, generator=r).bfloat16().cuda()
    x, residual, go, gn = (some() for _ in range(4))
    big = lambda t: t.repeat(times, 1)
    w = (1 + 0.1 * torch.randn(d, generator=r)).cuda()
    X, R = big(x), big(residual)
    N = torch.empty_like(X)
    robe.robe_residual_forward(X, R, R, N, w, w, None, 0.5)  # (in place)
    assert same_bits(R[-block:], R[:block]) and same_bits(N[-block:], N[:block])
    small, normed = torch.empty_like(x), torch.empty_like(x)
    robe.robe_residual_forward(x, residual, small, normed, w, w, None, 0.5)
    assert same_bits(R[:block], small) and same_bits(N[-block:], normed)
    del N
    GO, GN, GX = big(go), big(gn), torch.empty_like(X)
    g1, g2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(block * times, d), dtype=torch.uint8, device="cuda")
    robe.robe_residual_backward(GO, GN, X, R, GX, GO, w, w, None, g1, g2, None, ws, 0.5)
    assert same_bits(GO[-block:], GO[:block]) and same_bits(GX[-block:], GX[:block])
    s1, s2, gx, gr = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    robe.robe_residual_backward(go, gn, x, small, gx, gr, w, w, None, s1, s2, None, ws, 0.5)
    assert same_bits(GX[:block], gx) and same_bits(GO[:block], gr)
    # sums over rows: a thread's chunk (148 CTAs at least share the rows) in fp32, the chunks' in 64 bits
    chain = (block * times / 148 + 64) * ref.U
    n1 = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    for all_rows, few, terms in ((g1, s1, 0.5 * gr.double() * n1), (g2, s2, gn.double() * normed.double() / w)):
        assert bool(((all_rows.double() - times * few.double()).abs() <= 2 * chain * times * terms.abs().sum(0)).all())


def test_bias_of_more_than_2_to_31_places():
    q = k = 47_000
    room(16)
    b = robe.robe_bias_create(32, 1000, False)
    rows = torch.randn(32, 1, generator=gen(6)).cuda()
    out = torch.empty(1, 1, q, k, dtype=torch.bfloat16, device="cuda")
    robe.robe_bias_forward(b, rows, out, 0, True)
    edges = torch.tensor(robe.robe_bias_get_edges(b)[1:], device="cuda")
    for i in (0, 1, 20_000, q - 2, q - 1):
        r = torch.arange(k, device="cuda") - i
        want = torch.where(r > 0, -math.inf, rows[torch.bucketize((-r).clamp(min=0), edges, right=True), 0]).bfloat16()
        assert same_bits(out[0, 0, i], want), i
    # of ones: the number of places of every bucket, exact in 64 bits and rounded once; in fp32 sums of up to 64 ones are exact
    out.fill_(1.0)
    got = torch.empty(32, 1, device="cuda")
    ws = torch.empty(robe.robe_bias_backward_workspace_bytes(b, 1, 1, q, k), dtype=torch.uint8, device="cuda")
    robe.robe_bias_backward(b, out, got, ws, 0, True)
    dist = torch.arange(q, device="cuda")
    want = torch.zeros(32, dtype=torch.float64, device="cuda")
    want.index_add_(0, torch.bucketize(dist, edges, right=True), (q - dist).double())
    assert torch.equal(got[:, 0], want.float())
    robe.robe_bias_destroy(b)


@pytest.mark.parametrize("rows,d,scale", [(148 * 16 * 2000, 264, 1.01922607421875), (148 * 1600, 8200, 1.27313232421875)])
def test_residual_sums_of_many_rows(rows, d, scale):
    # ones without eps, all terms are the scale: a single sum of 1600 of this one in fp32 is off by 400 U, of 2000 of that by 500 U.
    # 256 rows in fp32 (256 U), the rest in 64 bits, one rounding of the sum, one of a gate's scale
    room(3 * rows * d * 4 >> 30)
    x = torch.ones(rows, d, device="cuda")
    gx, w, gate = torch.empty_like(x), torch.ones(d, device="cuda"), torch.ones(4, d, device="cuda")
    for gates in (0, 4):
        gw, gg = torch.empty(d, device="cuda"), torch.empty_like(gate)
        ws = torch.empty(robe.robe_residual_backward_workspace_bytes(rows, d, gates), dtype=torch.uint8, device="cuda")
        robe.robe_residual_backward(x, None, x, None, gx, None, w, None, gate if gates else None, gw, None, gg if gates else None, ws,
                                    scale, 0, 0.0)
        for got, terms in [(gw, rows)] + ([(gg, rows // 4)] if gates else []):
            off = (got.double() - terms * scale).abs().max() / (terms * scale)
            assert off <= 258 * ref.U, (gates, terms, float(off) / ref.U)


@pytest.mark.parametrize("dtype", TYPES)
def test_bias_of_long_rows(dtype):
    # several CTAs along a row, both ways, and a gradient whose diagonals are cut in chunks
    b = robe.robe_bias_create(16, 200, True)
    for q, k, start in [(2, 70_001, 69_000), (40, 30_000, 15_000), (6, 25_003, 30_000)]:
        rows, index = bias_case(2, q, k, (16, 200, True), False, [start], dtype)
        out = torch.empty(1, 2, q, k, dtype=dtype, device="cuda")
        robe.robe_bias_forward(b, rows.cuda(), out, start)
        assert same_bits(out.cpu(), rows[index].permute(0, 3, 1, 2).to(dtype))
        g = torch.randn(1, 2, q, k, generator=gen(q)).to(dtype)
        want, bound = bias_grad_reference(g, index, 16)
        got = torch.empty(16, 2, device="cuda")
        ws = Workspace(robe.robe_bias_backward_workspace_bytes(b, 2, 1, q, k))
        robe.robe_bias_backward(b, g.cuda(), got, ws.own, start)
        ref.assert_within(got, want, bound, (q, k))
        assert ws.kept_within()
    robe.robe_bias_destroy(b)


# ---------------------------------------------------------------- streams, graphs, together


def test_both_ways_of_calling_give_the_same():
    # numbers that the native path leaves to ctypes (numpy's), and plain ones
    import numpy as np
    x, y = torch.randn(60, 200, generator=gen(1)).cuda(), torch.randn(60, 200, generator=gen(2)).cuda()
    w = torch.randn(200, generator=gen(3)).cuda()
    gate = torch.randn(20, 200, generator=gen(4)).cuda()
    b = robe.robe_bias_create(32, 128, False)
    rows, start = torch.randn(32, 3, generator=gen(5)).cuda(), torch.tensor([5, 70], device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    results = []
    for number, truth in ((float, bool), (np.float64, int)):
        got = [torch.full_like(x, NAN) for _ in range(5)]
        gg, g1, g2 = torch.full_like(gate, NAN), torch.full_like(w, NAN), torch.full_like(w, NAN)
        robe.robe_dropout(x, got[0], number(0.25), 7, 8)
        robe.robe_residual_forward(x, y, got[1], got[2], w, w, gate, number(0.5), 1, 1e-5, 0.1, 2, 3)
        robe.robe_residual_backward(y, x, x, got[1], got[3], got[4], w, w, gate, g1, g2, gg, ws, number(0.5), 1, 1e-5, 0.1, 2, 3)
        bias, grad_rows = torch.full((2, 3, 40, 90), NAN, device="cuda"), torch.full_like(rows, NAN)
        robe.robe_bias_forward(b, rows, bias, start, truth(1))
        robe.robe_bias_backward(b, bias.nan_to_num(neginf=1.0), grad_rows, ws, start, truth(1))
        results.append(got + [gg, g1, g2, bias, grad_rows])
    assert all(same_bits(p, q) for p, q in zip(*results))
    assert not any(t.isnan().any() for t in results[0])
    robe.robe_bias_destroy(b)


@pytest.mark.parametrize("rows,d", [(5000, 4096), (40_000, 128), (300, 12_288)])
def test_large_calls_are_captured(rows, d):
    x, y = (torch.randn(rows, d, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(d, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    out, normed, gx, gr = (torch.empty_like(x) for _ in range(4))
    g1, g2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(robe.robe_residual_backward_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")

    def both():
        robe.robe_residual_forward(x, y, out, normed, w, w, None, 0.5, 0, 1e-6, 0.1, 5, 6, step)
        robe.robe_residual_backward(y, x, x, out, gx, gr, w, w, None, g1, g2, None, ws, 0.5, 0, 1e-6, 0.1, 5, 6, step)

    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, normed, gx, gr, g1, g2)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for t in (out, normed, gx, gr, g1, g2):
        t.fill_(NAN)
    g.replay()
    torch.cuda.synchronize()
    assert all(same_bits(a, b) for a, b in zip(want, (out, normed, gx, gr, g1, g2)))
    del g


def test_two_streams_at_once_on_one_handle():
    b = robe.robe_bias_create(32, 128, True)
    g = [torch.randn(2, 4, 300, 300, generator=gen(n)).cuda() for n in range(2)]
    size = robe.robe_bias_backward_workspace_bytes(b, 4, 2, 300, 300)
    alone = []
    for t in g:
        got = torch.empty(32, 4, device="cuda")
        robe.robe_bias_backward(b, t, got, torch.empty(size, dtype=torch.uint8, device="cuda"))
        alone.append(got)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [torch.empty(32, 4, device="cuda") for _ in g]
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in g]
    torch.cuda.synchronize()
    for _ in range(20):
        for n in range(2):
            robe.robe_bias_backward(b, g[n], got[n], ws[n], 0, False, streams[n])
    torch.cuda.synchronize()
    assert same_bits(got[0], alone[0]) and same_bits(got[1], alone[1])
    robe.robe_bias_destroy(b)


def test_refusals_of_the_binding():
    x = torch.zeros(4, 8, device="cuda")
    b = robe.robe_bias_create(32, 128, False)
    bias = torch.zeros(1, 4, 8, 8, device="cuda")
    cases = [
        (ValueError, lambda: robe.robe_dropout(x, x[:2], 0.1, 1)),
        (ValueError, lambda: robe.robe_dropout(x.t(), x.t(), 0.1, 1)),
        (TypeError, lambda: robe.robe_dropout(x.half(), x.half(), 0.1, 1)),
        (TypeError, lambda: robe.robe_dropout(x, x.bfloat16(), 0.1, 1)),
        (TypeError, lambda: robe.robe_dropout(x, x, 0.1, 1, 0, torch.zeros(1, device="cuda"))),
        (robe.RobeError, lambda: robe.robe_dropout(x, x, 1.5, 1)),
        (ValueError, lambda: robe.robe_dropout(x[:1].expand(4, 8), x, 0.1, 1)),
        (ValueError, lambda: robe.robe_bias_forward(b, x, bias)),                                  # 4 rows for 32 buckets
        (ValueError, lambda: robe.robe_bias_forward(b, torch.zeros(32, 5, device="cuda"), bias)),  # 5 heads for 4
        (ValueError, lambda: robe.robe_bias_forward(b, torch.zeros(32, 8, device="cuda"), x)),
        (ValueError, lambda: robe.robe_bias_forward(b, torch.zeros(32, 4, device="cuda"), bias, torch.zeros(2, dtype=torch.int64, device="cuda"))),
        (TypeError, lambda: robe.robe_bias_forward(b, torch.zeros(32, 4, device="cuda"), bias, torch.zeros(1, dtype=torch.int32, device="cuda"))),
        (robe.RobeError, lambda: robe.robe_bias_backward(b, bias, torch.zeros(32, 4, device="cuda"), None)),
        (ValueError, lambda: robe.robe_residual_forward(x, None, torch.zeros_like(x), gate=torch.zeros(3, 8, device="cuda"))),
        (ValueError, lambda: robe.robe_residual_forward(x, None, torch.zeros_like(x), w_post=torch.zeros(7, device="cuda"))),
        (robe.RobeError, lambda: robe.robe_residual_forward(x, None, x)),
        (robe.RobeError, lambda: robe.robe_residual_forward(x, None, torch.zeros_like(x), torch.zeros_like(x))),
        (ValueError, lambda: robe.robe_residual_backward(x, None, x, None, torch.zeros_like(x), grad_gate=x)),
    ]
    for n, (error, call) in enumerate(cases):
        with pytest.raises(error):
            call()
            pytest.fail(f"case {n} was taken")
    torch.cuda.synchronize()
    robe.robe_bias_destroy(b)


def test_numbers_beyond_the_c_abis_are_refused():
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    b = robe.robe_bias_create(32, 128, False)
    bias, rows = torch.full((1, 4, 8, 8), NAN, device="cuda"), torch.zeros(32, 4, device="cuda")
    ws = torch.empty(robe.robe_bias_backward_workspace_bytes(b, 4, 1, 8, 8), dtype=torch.uint8, device="cuda")
    for start in (2**63, -2**63 - 1, 2**64 + 5):
        with pytest.raises(ValueError):
            robe.robe_bias_forward(b, rows, bias, start)
        with pytest.raises(ValueError):
            robe.robe_bias_backward(b, bias, rows, ws, start)
    assert bias.isnan().all()
    for norm in (2, -1, 2**32, 2**32 + 1, 2**64):
        with pytest.raises(robe.RobeError):
            robe.robe_residual_forward(x, None, torch.zeros_like(x), w_post=w, norm=norm)
    for start in (2**63 - 1, -2**63):  # the last ones that there are
        robe.robe_bias_forward(b, rows, bias, start)
        assert not bias.any()
    robe.robe_bias_destroy(b)


def test_calls_on_another_stream():
    side = torch.cuda.Stream()
    x = torch.randn(3000, 128, generator=gen(1)).cuda()
    torch.cuda.synchronize()
    out = torch.empty_like(x)
    with torch.cuda.stream(side):
        robe.robe_dropout(x, out, 0.25, 1, 2)
    robe.robe_dropout(out, out, 0.0, 1, 2, None, side)  # a stream by name
    side.synchronize()
    assert same_bits(out.cpu(), dropped(x.cpu(), 0.25, 1, 2))


def model_step(s):
    """Lookup, dropout, norm, a block (here: a fixed product per row) joined again, the bias of an attention from the same
    array, and all gradients down to the array."""
    h, hb, b = s["h"], s["hb"], s["bias"]
    B, T, d, H, Q = s["B"], s["T"], s["d"], s["H"], s["Q"]
    robe.robe_forward(h, s["ids"], None, B, s["rows"])
    robe.robe_residual_forward(s["rows"], None, s["h0"], s["n0"], None, s["w0"], p=0.1, seed=5, offset=1, step=s["step"])
    torch.mul(s["n0"], 0.5, out=s["block"])
    robe.robe_residual_forward(s["block"], s["h0"], s["h1"], s["n1"], s["w1"], s["w2"], s["gate"], 0.5, robe.ROBE_NORM_LAYER, 1e-6,
                               0.1, 5, 2, s["step"])
    robe.robe_forward(hb, s["bucket_ids"], None, 32, s["bucket_rows"])
    robe.robe_bias_forward(b, s["bucket_rows"][:, 0], s["scores"], 0, True)
    # back
    s["grad"].zero_()
    robe.robe_bias_backward(b, s["g_scores"], s["g_bucket_rows"][:, 0], s["ws_bias"], 0, True)
    robe.robe_backward(hb, s["g_bucket_rows"], s["bucket_ids"], None, 32, s["grad"], 0.0, s["ws_b"])
    robe.robe_residual_backward(s["g_h1"], s["g_n1"], s["block"], s["h1"], s["g_block"], s["g_h0"], s["w1"], s["w2"], s["gate"],
                                s["g_w1"], s["g_w2"], s["g_gate"], s["ws"], 0.5, robe.ROBE_NORM_LAYER, 1e-6, 0.1, 5, 2, s["step"])
    torch.mul(s["g_block"], 0.5, out=s["g_n0"])
    robe.robe_residual_backward(s["g_h0"], s["g_n0"], s["rows"], s["h0"], s["g_rows"], None, None, s["w0"], None, None, s["g_w0"],
                                None, s["ws"], p=0.1, seed=5, offset=1, step=s["step"])
    robe.robe_backward(h, s["g_rows"], s["ids"], None, B, s["grad"], 0.0, s["ws_h"])
    s["step"].add_(1)


RESULTS = ["h1", "n1", "scores", "grad", "g_w0", "g_w1", "g_w2", "g_gate"]


def model_state(array=None):
    r = gen(11)
    B, T, d, H, Q, M = 48, 5, 64, 4, 70, 5000
    s = dict(B=B, T=T, d=d, H=H, Q=Q)
    rnd = lambda *shape: torch.randn(*shape, generator=r).cuda()
    s["array"] = rnd(M)
    s["h"], s["hb"] = robe.robe_create(M, 16, d, T, 3), robe.robe_create(M, 4, H, 1, 4)
    for h in (s["h"], s["hb"]):
        robe.robe_attach_array(h, s["array"])
        robe.robe_set_option(h, robe.ROBE_OPT_BWD_MODE, robe.ROBE_BWD_DETERMINISTIC)
    s["bias"] = robe.robe_bias_create(32, 64, False)
    s["ids"] = torch.randint(1000, (B * T,), generator=r).cuda()
    s["bucket_ids"] = torch.arange(32).cuda()
    for name in ("rows", "h0", "n0", "block", "h1", "n1", "g_block", "g_h0", "g_n0", "g_rows"):
        s[name] = torch.full((B, T, d), NAN).cuda()
    for name in ("w0", "w1", "w2"):
        s[name] = 1 + 0.1 * rnd(d)
        s["g_" + name] = torch.full((d,), NAN).cuda()
    s["gate"], s["g_gate"] = rnd(B, T, 1), torch.full((B, T, 1), NAN).cuda()
    s["bucket_rows"], s["g_bucket_rows"] = torch.full((32, 1, H), NAN).cuda(), torch.full((32, 1, H), NAN).cuda()
    s["scores"], s["g_scores"] = torch.full((2, H, Q, Q), NAN).cuda(), rnd(2, H, Q, Q)
    s["g_h1"], s["g_n1"] = rnd(B, T, d), rnd(B, T, d)
    s["grad"] = torch.zeros(M).cuda()
    s["step"] = torch.zeros(1, dtype=torch.int64).cuda()
    byte = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    s["ws"] = byte(robe.robe_residual_backward_workspace_bytes(B * T, d, 0))
    s["ws_bias"] = byte(robe.robe_bias_backward_workspace_bytes(s["bias"], H, 2, Q, Q))
    s["ws_h"] = byte(robe.robe_backward_workspace_bytes(s["h"], B, B * T))
    s["ws_b"] = byte(robe.robe_backward_workspace_bytes(s["hb"], 32, 32))
    return s


def close(s):
    torch.cuda.synchronize()
    robe.robe_destroy(s["h"])
    robe.robe_destroy(s["hb"])
    robe.robe_bias_destroy(s["bias"])


def test_a_models_rows_from_lookup_to_gradient_array():
    s = model_state()
    B, T, d, H, Q = (s[k] for k in ("B", "T", "d", "H", "Q"))
    model_step(s)
    torch.cuda.synchronize()
    host = lambda name: s[name].cpu().double()
    flat = lambda name: host(name).reshape(B * T, d)
    drop = lambda offset: ref.kept(B * T, d, 0.1, 5, offset).double() * ref.drop_scale(0.1)
    # each operator on what the one before it left in memory
    (h0, e0), (n0, en0) = ref.join(flat("rows"), None, None, host("w0"), None, 1.0, 0, 1e-6, drop(1))
    ref.assert_within(s["h0"].reshape(B * T, d), h0, e0, "h0")
    ref.assert_within(s["n0"].reshape(B * T, d), n0, en0, "n0")
    gate = host("gate").reshape(B * T, 1)
    (h1, e1), (n1, en1) = ref.join(flat("block"), flat("h0"), host("w1"), host("w2"), gate, 0.5, 1, 1e-6, drop(2))
    ref.assert_within(s["h1"].reshape(B * T, d), h1, e1, "h1")
    ref.assert_within(s["n1"].reshape(B * T, d), n1, en1, "n1")
    index = ref.bias_index(Q, Q, 0, 32, 64, False, True)
    want = torch.where((index < 0)[..., None], -math.inf, s["bucket_rows"].cpu()[:, 0][index.clamp(min=0)]).permute(2, 0, 1)
    assert same_bits(s["scores"].cpu(), want.expand(2, -1, -1, -1).contiguous())
    g = ref.join_grad(flat("g_h1"), flat("g_n1"), flat("block"), flat("h1"), host("w1"), host("w2"), gate, 0.5, 1, 1e-6, drop(2))
    for name, of in (("g_block", "x"), ("g_h0", "residual")):
        ref.assert_within(s[name].reshape(B * T, d), *g[of], name)
    for name, of in (("g_w1", "w_post"), ("g_w2", "w_pre"), ("g_gate", "gate")):
        ref.assert_within(s[name], g[of][0].reshape(s[name].shape), g[of][1].reshape(s[name].shape), name)
    g = ref.join_grad(flat("g_h0"), flat("g_n0"), flat("rows"), flat("h0"), None, host("w0"), None, 1.0, 0, 1e-6, drop(1))
    ref.assert_within(s["g_rows"].reshape(B * T, d), *g["x"], "g_rows")
    ref.assert_within(s["g_w0"], *g["w_pre"], "g_w0")
    want, bound = bias_grad_reference(s["g_scores"].cpu(), index[None].expand(2, -1, -1), 32)
    ref.assert_within(s["g_bucket_rows"][:, 0], want, bound, "g_bucket_rows")
    # and the array's gradient holds every row's and bucket row's mass (without the sign hash the scatter keeps sums)
    total = host("g_rows").sum() + host("g_bucket_rows").sum()
    mass = host("g_rows").abs().sum() + host("g_bucket_rows").abs().sum()
    assert abs(host("grad").sum() - total) <= 64 * ref.U * mass  # (a slot sums at most some dozens of terms)
    close(s)


def test_a_captured_step_replays_with_new_draws_beside_another_graph():
    # eager steps, then the same from two captured graphs that take turns and share their workspaces
    s = model_state()
    eager = []
    for _ in range(6):
        model_step(s)
        torch.cuda.synchronize()
        eager.append({k: s[k].clone() for k in RESULTS})
    assert not torch.equal(eager[0]["h1"], eager[1]["h1"])  # the step counter draws anew
    s["step"].zero_()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for g in graphs:
        with torch.cuda.graph(g, stream=side):
            model_step(s)
    torch.cuda.synchronize()
    s["step"].zero_()
    for n in range(6):
        for k in RESULTS:
            s[k].fill_(0.0 if k == "grad" else NAN)
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        for k in RESULTS:
            assert same_bits(s[k], eager[n][k]), (n, k)
    del graphs
    close(s)
