"""The lookup in a plain table and its gradient on the GPU against their definitions: types, odd sizes, strides, ids outside the
table, ids that repeat in every way that the sums are cut by, other streams, captured graphs."""
import math

import pytest
import torch

import paper_2108_02191_b200 as robe
import rows8_reference as ref
from test_gpu_row_ops import NAN, TYPES, Workspace, blank, gen, place, same_bits, surroundings_kept

pytestmark = pytest.mark.gpu


def ids_of(kind, n, vocab, seed=0):
    g = gen(seed)
    if kind == "uniform":
        return torch.randint(0, vocab, (n,), generator=g)
    if kind == "same":
        return torch.full((n,), vocab - 1)
    if kind == "distinct":
        return torch.randperm(vocab, generator=g)[:n] if n <= vocab else torch.arange(n) % vocab
    if kind == "few":  # frequent ones and rare ones
        return (torch.rand(n, generator=g) ** 4 * vocab).long().clamp(max=vocab - 1)
    if kind == "outside":  # half of them no row
        ids = torch.randint(0, vocab, (n,), generator=g)
        bad = torch.tensor([-1, vocab, 2**31 - 1, -2**31])[torch.randint(0, 4, (n,), generator=g)]
        return torch.where(torch.rand(n, generator=g) < 0.5, ids, bad)
    if kind == "none":
        return torch.full((n,), -1)
    raise AssertionError(kind)


# ---------------------------------------------------------------- lookup


@pytest.mark.parametrize("how", ["plain", "slice", "odd"])
@pytest.mark.parametrize("table_type", TYPES)
@pytest.mark.parametrize("out_type", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 5, 4096), (16, 1000, 64), (37, 50, 7), (129, 30, 100), (1000, 11, 12), (3, 9, 1001),
                                       (5000, 400, 128), (2, 3, 8200), (41_000, 900, 128), (7001, 300, 101), (700_001, 40, 1)])
def test_lookup(n, vocab, d, table_type, out_type, how):
    table = torch.randn(vocab, d, generator=gen(d)).to(table_type)
    ids = ids_of("outside" if n > 2 else "uniform", n, vocab)
    scale = math.sqrt(d)
    for kind in (torch.int64, torch.int32):
        out = blank((n, d), out_type, how)
        robe.robe_table_forward(place(table, how), ids.to(kind).cuda(), out, scale)
        inside = (ids >= 0) & (ids < vocab)
        want = (table[ids.clamp(0, vocab - 1)].float() * torch.tensor(scale, dtype=torch.float32)).to(out_type)
        want[~inside] = 0
        assert same_bits(out.cpu(), want) and surroundings_kept(out)


def test_lookup_of_ids_beyond_32_bits_and_of_nothing():
    table = torch.randn(4, 8, generator=gen(1)).cuda()
    ids = torch.tensor([2**32 + 1, 2**40, -2**63, 2**63 - 1, 3], device="cuda")
    out = blank((5, 8), torch.float32)
    robe.robe_table_forward(table, ids, out)
    assert not out[:4].any() and torch.equal(out[4], table[3])
    robe.robe_table_forward(table, ids[:0], out[:0])
    robe.robe_table_forward(table[:0], ids, out)  # no rows: every id is outside
    assert not out.any()
    out = blank((2, 3, 8), torch.float32)
    robe.robe_table_forward(table, torch.tensor([[0, 1, 2], [3, 3, -1]], device="cuda"), out)
    assert torch.equal(out[0], table[:3]) and torch.equal(out[1, :2], table[[3, 3]]) and not out[1, 2].any()


def test_lookup_keeps_what_is_not_a_number():
    table = torch.tensor([[NAN, math.inf, -math.inf, 0.0, -0.0, 1e-45, 3.4e38, -1.0]])
    out = blank((1, 8), torch.float32)
    robe.robe_table_forward(table.cuda(), torch.zeros(1, dtype=torch.int64, device="cuda"), out, 1.0)
    assert out[0, 0].isnan() and torch.equal(out[0, 1:].cpu(), table[0, 1:])


@pytest.mark.parametrize("dtype", TYPES)
def test_lookup_past_2_to_31_elements(dtype):
    d = 1024
    vocab = n = 2**31 // d + 77
    if torch.cuda.mem_get_info()[0] < 2 * n * d * dtype.itemsize + (4 << 30):
        pytest.skip("not enough memory")
    table = torch.arange(vocab, device="cuda").remainder(251).to(dtype)[:, None].expand(vocab, d).contiguous()
    ids = torch.arange(n - 1, -1, -1, device="cuda")
    out = torch.empty(n, d, dtype=dtype, device="cuda")
    robe.robe_table_forward(table, ids, out, 2.0)
    want = (2 * ids.remainder(251)).to(dtype)
    for c in (0, 511, d - 1):
        assert torch.equal(out[:, c], want)


# ---------------------------------------------------------------- gradient


def whole(n, d, most, seed, dtype):
    """Whole numbers whose sums are exact."""
    return torch.randint(-most, most + 1, (n, d), generator=gen(seed)).to(dtype)


SIZES = [(1, 1, 1), (1, 3, 64), (2, 2, 3), (15, 4, 8), (16, 4, 8), (17, 4, 8), (33, 700, 100), (64, 5, 1001), (257, 2, 130), (1000, 300, 7),
         (4096, 100, 16), (5003, 2000, 36), (300, 4, 4100), (20_000, 3, 5), (3000, 70_000, 12)]
# around the sizes at which the ids are sorted in another way, and with runs of many chunks
SORTS = [(512, 600, 9), (513, 600, 9), (1024, 2, 4), (1025, 40_000, 4), (8192, 7, 8), (8193, 300, 8), (16_385, 5000, 3), (32_768, 2**20, 2), (32_769, 90, 4),
         (65_536, 1, 4), (65_537, 20, 4), (70_001, 3000, 8), (200_000, 2, 6)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "same", "distinct", "few", "outside", "none"])
@pytest.mark.parametrize("n,vocab,d", SIZES)
def test_gradient_of_whole_numbers(n, vocab, d, kind, dtype, how, accumulate):
    # sums of whole numbers below 2^24: exact in any order, so every bit is known
    grad, ids = whole(n, d, 7, n + d, dtype), ids_of(kind, n, vocab, d)
    old = whole(vocab, d, 100, 5, torch.float32) / 4
    table = place(old, how) if accumulate else blank((vocab, d), torch.float32, how)
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    index = ids.to(torch.int32 if n % 2 else torch.int64).cuda()
    robe.robe_table_backward(place(grad, how), index, table, ws.own, 0.5, accumulate)
    s, _ = ref.table_sums(grad, ids, vocab)
    want = (0.5 * s + (old.double() if accumulate else 0.0)).float()
    assert torch.equal(table.cpu(), want) and surroundings_kept(table) and ws.kept_within()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["uniform", "same", "few", "outside"])
@pytest.mark.parametrize("n,vocab,d", SORTS)
def test_gradient_of_many_ids(n, vocab, d, kind, accumulate):
    test_gradient_of_whole_numbers(n, vocab, d, kind, torch.bfloat16, "plain", accumulate)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,d,kind", [(5003, 900, 100, "few"), (100_000, 50, 64, "few"), (20_000, 3, 256, "same"), (2000, 5000, 1000, "uniform")])
def test_gradient_of_any_numbers(n, vocab, d, kind, dtype):
    # fp32 sums of at most 256 terms: off by at most 255 half steps of the terms' magnitudes, whatever they meet; joined in
    # 64 bits, rounded to fp32 (once more by the scale, once by the sum with what is there)
    grad, ids = torch.randn(n, d, generator=gen(n)).to(dtype), ids_of(kind, n, vocab)
    old, scale = torch.randn(vocab, d, generator=gen(3)), 0.3
    s, l1 = ref.table_sums(grad, ids, vocab)
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    half = 2.0 ** -24
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    for accumulate in (False, True):
        table = old.cuda() if accumulate else blank((vocab, d), torch.float32)
        robe.robe_table_backward(grad.cuda(), ids.cuda(), table, ws.own, scale, accumulate)
        want = scale32 * s + (old.double() if accumulate else 0.0)
        most = 256 * half * scale32 * l1 + 2 * half * want.abs() + 2.0 ** -140
        assert ((table.cpu().double() - want).abs() <= most).all()
        again = old.cuda() if accumulate else blank((vocab, d), torch.float32)
        robe.robe_table_backward(grad.cuda(), ids.cuda(), again, ws.own, scale, accumulate)
        assert same_bits(again, table)  # the same call, the same bits


@pytest.mark.parametrize("n,d", [(300_000, 4096), (2_000_000, 100)])
def test_gradient_in_longer_chunks(n, d):
    # sizes whose chunks are longer than the shortest; ids in runs of every length around the chunks' borders
    vocab = 5000
    if torch.cuda.mem_get_info()[0] < 10 << 30:
        pytest.skip("not enough memory")
    g = torch.Generator(device="cuda").manual_seed(1)
    grad = torch.randint(-3, 4, (n, d), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    ids = (torch.rand(n, generator=g, device="cuda") ** 6 * vocab).long().clamp(max=vocab - 1)
    table = torch.full((vocab, d), NAN, device="cuda")
    ws = torch.empty(robe.robe_table_backward_workspace_bytes(n, vocab, d), dtype=torch.uint8, device="cuda")
    robe.robe_table_backward(grad, ids, table, ws)
    for c in (0, 1, d // 2, d - 1):
        want = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, ids, grad[:, c].double())
        assert torch.equal(table[:, c].double(), want)


@pytest.mark.parametrize("n,largest,d", [(75_776, 79_000, 128), (151_552, 157_000, 64), (9472, 10_000, 1024), (2368, 2500, 4096), (16, 2369, 4096)])
def test_gradient_with_the_workspace_of_a_larger_call(n, largest, d):
    # calls of which the larger ones have fewer, longer chunks
    vocab = 50
    g = torch.Generator(device="cuda").manual_seed(n)
    grad = torch.randint(-3, 4, (n, d), generator=g, device="cuda").float()
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ws = Workspace(robe.robe_table_backward_workspace_bytes(largest, vocab, d))
    table = torch.full((vocab, d), NAN, device="cuda")
    robe.robe_table_backward(grad, ids, table, ws.own)
    want = torch.zeros(vocab, d, device="cuda").index_add_(0, ids, grad)  # (whole numbers: exact in any order)
    assert torch.equal(table, want) and ws.kept_within()


def test_gradient_skips_one_id_and_keeps_rows_without_ids():
    n, vocab, d = 500, 40, 24
    ids = torch.randint(0, 20, (n,), generator=gen(1))
    grad = whole(n, d, 5, 2, torch.float32)
    old = torch.randn(vocab, d, generator=gen(3))
    old[25, 3], old[26, 4], old[7, 0] = NAN, math.inf, -0.0
    table = old.cuda()
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    robe.robe_table_backward(grad.cuda(), ids.cuda(), table, ws.own, 1.0, True, 7)
    s, _ = ref.table_sums(grad, ids, vocab, 7)
    touched = torch.zeros(vocab, dtype=torch.bool)
    touched[ids] = True
    touched[7] = False
    assert same_bits(table.cpu()[~touched], old[~touched])
    want = (s + old.double()).float()
    assert torch.equal(table.cpu()[touched], want[touched])
    # written whole: +0 for the skipped one and for those without ids
    table = blank((vocab, d), torch.float32)
    robe.robe_table_backward(grad.cuda(), ids.cuda(), table, ws.own, 1.0, False, 7)
    assert torch.equal(table.cpu(), s.float()) and not torch.signbit(table[~touched.cuda()]).any()


def test_gradient_of_nothing():
    table = blank((5, 9), torch.float32)
    ws = Workspace(robe.robe_table_backward_workspace_bytes(0, 5, 9))
    none = torch.empty(0, 9, device="cuda")
    robe.robe_table_backward(none, torch.empty(0, dtype=torch.int64, device="cuda"), table, ws.own)
    assert torch.equal(table, torch.zeros_like(table))
    table.fill_(3.0)
    robe.robe_table_backward(none, torch.empty(0, dtype=torch.int64, device="cuda"), table, ws.own, 1.0, True)
    assert (table == 3.0).all()


def test_gradient_of_what_is_not_a_number_stays_in_its_row():
    n, vocab, d = 400, 10, 40
    ids = torch.arange(n) % vocab
    grad = whole(n, d, 3, 1, torch.bfloat16)
    grad[13, 5], grad[27, 6] = NAN, math.inf
    table = blank((vocab, d), torch.float32)
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    robe.robe_table_backward(grad.cuda(), ids.cuda(), table, ws.own)
    s, _ = ref.table_sums(grad, ids, vocab)
    assert torch.equal(table.cpu().isnan(), s.isnan()) and int(s.isnan().sum()) == 1
    assert torch.equal(table.cpu().nan_to_num(7.0), s.float().nan_to_num(7.0))


def test_lookup_and_gradient_are_transposes():
    n, vocab, d, scale = 300, 77, 50, 0.25
    table, up = torch.randn(vocab, d, generator=gen(1)), torch.randn(n, d, generator=gen(2))
    ids = ids_of("outside", n, vocab)
    out, grad = blank((n, d), torch.float32), blank((vocab, d), torch.float32)
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    robe.robe_table_forward(table.cuda(), ids.cuda(), out, scale)
    robe.robe_table_backward(up.cuda(), ids.cuda(), grad, ws.own, scale)
    a, b = (out.double().cpu() * up.double()).sum(), (table.double() * grad.double().cpu()).sum()
    # either side: at most 16 terms a row of the gradient, one rounding a product
    assert abs(float(a - b)) <= 2.0 ** -24 * 20 * float((out.double().cpu() * up.double()).abs().sum())


def test_sgd_step_of_a_table():
    n, vocab, d = 1000, 60, 32
    table, up, ids = whole(vocab, d, 50, 1, torch.float32), whole(n, d, 4, 2, torch.bfloat16), ids_of("few", n, vocab)
    t = table.cuda()
    ws = Workspace(robe.robe_table_backward_workspace_bytes(n, vocab, d))
    robe.robe_table_backward(up.cuda(), ids.cuda(), t, ws.own, -0.25, True)
    s, _ = ref.table_sums(up, ids, vocab)
    assert torch.equal(t.cpu(), (table.double() - 0.25 * s).float())


def test_two_captured_steps_share_a_workspace():
    n, vocab, d = 700, 90, 48
    state = []
    side = torch.cuda.Stream()
    ws = torch.full((robe.robe_table_backward_workspace_bytes(n, vocab, d),), 0xA5, dtype=torch.uint8, device="cuda")
    for k in range(2):
        s = dict(table=torch.randn(vocab, d, generator=gen(k)).cuda(), ids=ids_of("few", n, vocab, k).cuda(),
                 up=whole(n, d, 3, k, torch.float32).cuda(), out=torch.empty(n, d, device="cuda"), grad=torch.empty(vocab, d, device="cuda"))
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            robe.robe_table_forward(s["table"], s["ids"], s["out"], 2.0)
            robe.robe_table_backward(s["up"], s["ids"], s["grad"], ws, 1.0)
        state.append((s, g))
    for turn in range(3):
        for k, (s, g) in enumerate(state):
            s["ids"].copy_(ids_of("uniform" if turn else "same", n, vocab, 10 * turn + k))
            s["grad"].fill_(NAN)
            g.replay()
            assert torch.equal(s["out"], s["table"][s["ids"]] * 2.0)
            want, _ = ref.table_sums(s["up"].cpu(), s["ids"].cpu(), vocab)
            assert torch.equal(s["grad"].cpu(), want.float())


def test_calls_on_two_streams_at_once():
    n, vocab, d = 20_000, 3000, 64
    streams = [torch.cuda.Stream() for _ in range(2)]
    ids = [ids_of("few", n, vocab, k).cuda() for k in range(2)]
    up = [whole(n, d, 3, k, torch.float32).cuda() for k in range(2)]
    grad = [torch.empty(vocab, d, device="cuda") for _ in range(2)]
    ws = [torch.empty(robe.robe_table_backward_workspace_bytes(n, vocab, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            robe.robe_table_backward(up[k], ids[k], grad[k], ws[k], 1.0, stream=streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        want, _ = ref.table_sums(up[k].cpu(), ids[k].cpu(), vocab)
        assert torch.equal(grad[k].cpu(), want.float())


def test_both_ways_of_calling_give_the_same(monkeypatch):
    n, vocab, d = 200, 31, 20
    table, up, ids = torch.randn(vocab, d, generator=gen(1)).cuda(), torch.randn(n, d, generator=gen(2)).cuda(), ids_of("few", n, vocab).cuda()
    ws = torch.empty(robe.robe_table_backward_workspace_bytes(n, vocab, d), dtype=torch.uint8, device="cuda")

    def both():
        out, grad = torch.empty(n, d, device="cuda"), torch.empty(vocab, d, device="cuda")
        robe.robe_table_forward(table, ids, out, 1.5)
        robe.robe_table_backward(up, ids, grad, ws, 0.5, False, 3)
        return out, grad

    a = both()
    assert robe.binding._native.table_forward(table, ids, torch.empty(n, d, device="cuda"), 1.5, None) == robe.ROBE_OK
    for name in ("table_forward", "table_backward"):
        monkeypatch.setattr(robe.binding._native, name, lambda *_: 1, raising=False)
    b = both()
    assert all(same_bits(x, y) for x, y in zip(a, b))


def test_refusals_of_the_binding():
    table, out, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    ws = torch.empty(robe.robe_table_backward_workspace_bytes(3, 4, 8), dtype=torch.uint8, device="cuda")
    for bad in [lambda: robe.robe_table_forward(table, ids.float(), out), lambda: robe.robe_table_forward(table, ids[:2], out),
                lambda: robe.robe_table_forward(table, ids, out[:, :7]), lambda: robe.robe_table_forward(table.half(), ids, out),
                lambda: robe.robe_table_forward(table, ids.cpu(), out), lambda: robe.robe_table_forward(table.t(), ids, out),
                lambda: robe.robe_table_backward(out, ids, table.bfloat16(), ws), lambda: robe.robe_table_backward(out, ids, table[:, :7], ws),
                lambda: robe.robe_table_backward(out, ids, table, ws, 1.0, False, 2**63),
                lambda: robe.robe_table_forward(table, torch.zeros(6, dtype=torch.int64, device="cuda")[::2], out)]:
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad, status in [(lambda: robe.robe_table_backward(out, ids, table, ws[:-256]), robe.ROBE_ERR_WORKSPACE),
                        (lambda: robe.robe_table_backward(out, ids, table, None), robe.ROBE_ERR_WORKSPACE),
                        (lambda: robe.robe_table_backward(out, ids, table, ws[8:]), robe.ROBE_ERR_WORKSPACE),
                        (lambda: robe.robe_table_forward(table, ids, table[:3]), robe.ROBE_ERR_INVALID_ARG),
                        (lambda: robe.robe_table_backward(table[:3], ids, table, ws), robe.ROBE_ERR_INVALID_ARG)]:
        with pytest.raises(robe.RobeError) as e:
            bad()
        assert e.value.status == status
