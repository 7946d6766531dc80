"""Plain tables and rows in 8 bits without a GPU: the definitions against independent statements of them, argument checks of the C ABI
and of the binding."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2108_02191_b200 as robe
import rows8_reference as ref

BAD = robe.ROBE_ERR_INVALID_ARG
WORK = robe.ROBE_ERR_WORKSPACE
P = [C.c_void_p(0x10000 + k * 0x1000000) for k in range(12)]  # never dereferenced


def lib():
    return robe.binding.raw()


# ---------------------------------------------------------------- the definitions


def test_e4m3_numbers():
    table = ref.e4m3_values()
    assert table[0] == 0 and table[1] == 2.0 ** -9 and table[8] == 2.0 ** -6 and table[126] == 448 and (np.diff(table) > 0).all()
    # torch's type names the same numbers
    theirs = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert (theirs == table).all()


def test_nearest_codes():
    table = ref.e4m3_values()
    assert (ref.nearest_e4m3(table) == np.arange(127)).all()
    middle = (table[1:] + table[:-1]) / 2
    codes = ref.nearest_e4m3(middle)
    assert (codes % 2 == 0).all() and (np.abs(codes.astype(int) - np.arange(126)) <= 1).all()  # ties go to the even code
    assert (ref.nearest_e4m3(-middle) == codes + 128).all()
    v = np.random.default_rng(1).uniform(-448, 448, 5000)
    back = np.where(ref.nearest_e4m3(v) > 127, -1, 1) * table[ref.nearest_e4m3(v) % 128]
    assert (np.abs(back - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10)).all()


def test_quantised_rows_by_hand():
    x = torch.tensor([[127.0, -254.0, 1.0, 63.5, 0.0, 0.0]])
    codes, scales = ref.quantize(x, 4, torch.int8)
    assert float(scales[0, 0]) == 2.0 and abs(float(scales[0, 1]) * 127 / 2.0 ** -90 - 1) <= 2.0 ** -24  # (a group of zeros)
    assert codes.view(torch.int8).tolist() == [[64, -127, 0, 32, 0, 0]]  # 63.5 and 31.75; 0.5 to the even 0
    codes, scales = ref.quantize(torch.tensor([[448.0, -17.0, 1.0, 0.0]]), 0, torch.float8_e4m3fn)
    assert scales.tolist() == [[1.0]] and codes.tolist() == [[126, 128 + 0x58, 0x38, 0]]  # 17 lies between 16 and 18: the even one


def test_places_of_a_cache():
    pages = torch.tensor([[4, 1], [0, -1]], dtype=torch.int32)
    assert ref.places(pages, 2, 5, 6, [0, 3, 5], [1, 0]) == [9, 2, 3, 0, 1, -2]
    assert ref.places(pages, 2, 4, 6, None, [1, 1]) == [-1, 2, 3, 1, -1, -1]


def test_attention_of_one_key():
    # one key: the result is its value, whatever the score
    q, k, v = torch.randn(2, 8).double(), torch.randn(1, 8).double(), torch.randn(1, 8).double()
    out, p = ref.attention(q, k, v)
    assert torch.allclose(out, v.expand(2, 8), rtol=0, atol=1e-15) and p.tolist() == [[1.0], [1.0]]


# ---------------------------------------------------------------- tables: argument checks


def forward(**o):
    a = dict(table=P[0], ld=8, vocab=100, d=8, type=robe.ROBE_F32, ids=P[1], index=robe.ROBE_I64, rows=4, scale=1.0, out=P[2], out_ld=8, out_type=robe.ROBE_F32)
    a.update(o)
    return lib().robe_table_forward(a["table"], a["ld"], a["vocab"], a["d"], a["type"], a["ids"], a["index"], a["rows"], a["scale"], a["out"], a["out_ld"],
                                    a["out_type"], None)


@pytest.mark.parametrize("o", [dict(table=None), dict(ids=None), dict(out=None), dict(type=2), dict(out_type=3), dict(index=2), dict(rows=-1), dict(vocab=-1),
                               dict(vocab=2**31), dict(d=0), dict(d=2**20 + 1), dict(ld=7), dict(out_ld=7), dict(ids=C.c_void_p(0x10004)), dict(table=C.c_void_p(0x10002)),
                               dict(out=P[0]), dict(out=P[1]), dict(rows=2**62), dict(rows=2**59), dict(index=robe.ROBE_I32, ids=C.c_void_p(0x10002))])
def test_lookup_refuses(o):
    assert forward(**o) == BAD


def test_lookup_of_nothing_launches_nothing():
    assert forward(rows=0, ids=None, out=None) == robe.ROBE_OK


def backward(**o):
    a = dict(grad=P[0], ld=8, type=robe.ROBE_F32, ids=P[1], index=robe.ROBE_I64, rows=4, scale=1.0, skip=-1, acc=0, table=P[2], table_ld=8, vocab=100, d=8, ws=P[3],
             bytes=1 << 40)
    a.update(o)
    return lib().robe_table_backward(a["grad"], a["ld"], a["type"], a["ids"], a["index"], a["rows"], a["scale"], a["skip"], a["acc"], a["table"], a["table_ld"],
                                     a["vocab"], a["d"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("o,status", [(dict(grad=None), BAD), (dict(ids=None), BAD), (dict(table=None), BAD), (dict(type=2), BAD), (dict(index=5), BAD), (dict(acc=2), BAD),
                                      (dict(rows=2**31), BAD), (dict(vocab=2**31), BAD), (dict(d=0), BAD), (dict(ld=4), BAD), (dict(table_ld=4), BAD),
                                      (dict(table=P[0]), BAD), (dict(ws=P[2]), BAD), (dict(ws=None), WORK), (dict(bytes=100), WORK), (dict(ws=C.c_void_p(0x7000010)), WORK)])
def test_table_gradient_refuses(o, status):
    assert backward(**o) == status


def test_workspace_of_the_table_gradient():
    need = robe.robe_table_backward_workspace_bytes
    for bad in [(-1, 5, 5), (5, -1, 5), (5, 5, 0), (2**31, 5, 5), (5, 2**31, 5), (5, 5, 2**20 + 1), (2**64, 5, 5)]:
        assert need(*bad) == 0
    assert backward(bytes=need(4, 100, 8) - 1) == WORK
    # ids and positions twice, a byte an id of the table, two rows of sums for 16 rows of the gradient
    # (there is no byte an id any more: the figure does not go by the table, and stays within the bound all the same)
    n, vocab, d = 16384, 65536, 4096
    assert need(n, vocab, d) <= 16 * n + vocab + n // 16 * 2 * d * 4 + 400_000
    # nothing overflows at the limits
    assert need(2**31 - 1, 2**31 - 1, 2**20) > 2**31 * 16
    # an fp32 sum has at most 256 rows: two rows of sums for every 256 at least
    assert need(10**6, 100, 8192) >= 10**6 // 256 * 2 * 8192 * 4


def test_workspace_of_the_table_gradient_never_falls_as_a_call_grows():
    # one sized for the largest batch serves every smaller one; chunks of rows get longer where a call has more than a wave of them
    need = robe.robe_table_backward_workspace_bytes
    for d in (1, 3, 4, 64, 100, 128, 1000, 1024, 4096, 4099, 8192, 2**20):
        for rows in (range(0, 3000), range(9000, 12_000), range(65_000, 66_000), range(75_000, 80_000, 3), range(150_000, 160_000, 7), range(0, 3_000_000, 1237),
                     range(2**31 - 9000, 2**31, 11)):
            sizes = [need(n, 10**6, d) for n in rows]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), (d, rows)
    for n in (1, 16, 17, 149, 512, 5003, 16_384, 65_536, 65_537, 100_000, 2 * 10**6, 2**31 - 1):
        sizes = [need(n, 10**6, d) for d in list(range(1, 9000)) + list(range(9000, 2**20 + 1, 997))]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), n
    # sizes at which it fell: the row counts at which chunks become longer
    for n, d in [(75_776, 128), (151_552, 64), (9472, 1024), (2368, 4096)]:
        assert need(n + 1, 10**6, d) >= need(n, 10**6, d)
    # a call with the workspace of a larger one; one byte less than its own is refused (checked before anything is launched)
    for n, d in [(75_777, 128), (2369, 4096)]:
        assert backward(rows=n, vocab=10**6, d=d, ld=d, table_ld=d, grad=C.c_void_p(1 << 40), ids=C.c_void_p(2 << 40), table=C.c_void_p(3 << 40), ws=C.c_void_p(4 << 40),
                        bytes=need(n, 10**6, d) - 1) == WORK


# ---------------------------------------------------------------- rows in 8 bits: argument checks


def quantize(**o):
    a = dict(rows=4, d=64, type=robe.ROBE_F32, norm=0, eps=1e-6, scale=1.0, x=P[0], x_ld=64, res=P[1], res_ld=64, w=P[2], out=P[3], out_ld=64, codes=P[4], codes_ld=64,
             code=robe.ROBE_E4M3, group=32, scales=P[5], scales_ld=2)
    a.update(o)
    return lib().robe_residual_quantize(a["rows"], a["d"], a["type"], a["norm"], a["eps"], a["scale"], a["x"], a["x_ld"], a["res"], a["res_ld"], a["w"], a["out"],
                                        a["out_ld"], a["codes"], a["codes_ld"], a["code"], a["group"], a["scales"], a["scales_ld"], None)


@pytest.mark.parametrize("o", [dict(rows=-1), dict(rows=2**32 + 1), dict(d=0), dict(d=2**20 + 1), dict(type=2), dict(norm=2), dict(eps=-1.0), dict(eps=math.nan),
                               dict(eps=math.inf), dict(code=0), dict(code=4), dict(group=-1), dict(group=300, d=512, x_ld=512, res_ld=512, out_ld=512, codes_ld=512),
                               dict(x=None), dict(codes=None), dict(scales=None), dict(x_ld=63), dict(codes_ld=63), dict(scales_ld=1), dict(out=P[0]), dict(codes=P[0]),
                               dict(scales=P[4]), dict(w=C.c_void_p(0x10002)), dict(scales=C.c_void_p(0x10002)), dict(out=P[1], out_ld=65)])
def test_join_in_8_bits_refuses(o):
    assert quantize(**o) == BAD


def test_join_in_8_bits_of_nothing():
    assert quantize(rows=0, x=None, res=None, out=None, codes=None, scales=None) == robe.ROBE_OK


def cache(**o):
    a = dict(codes=P[0], codes_ld=64, codes_page=64 * 16, scales=P[1], scales_ld=2, scales_page=32, num_pages=10, page_rows=16, d=64, group=32, code_type=robe.ROBE_I8,
             pages=P[2], pages_ld=3, batch=2, max_pages=3, offsets=None, starts=None)
    a.update(o)
    return robe.binding._Cache(**{k: (v.value if isinstance(v, C.c_void_p) else v) for k, v in a.items()})


CACHE_BAD = [dict(codes=None), dict(scales=None), dict(pages=None), dict(codes_ld=63), dict(codes_page=64 * 16 - 1), dict(scales_page=31), dict(num_pages=-1),
             dict(num_pages=2**31), dict(page_rows=0), dict(page_rows=2**31), dict(d=0), dict(group=-1), dict(code_type=1), dict(batch=-1), dict(max_pages=-1), dict(pages_ld=2),
             dict(scales=P[0]), dict(pages=C.c_void_p(0x10002)), dict(offsets=C.c_void_p(0x9000004)), dict(starts=C.c_void_p(0x9000004)), dict(codes_ld=2**62)]


@pytest.mark.parametrize("o", CACHE_BAD)
def test_cache_calls_refuse(o):
    c = cache(**o)
    if o != dict(scales=P[0]):  # (two things that are read may be the same memory)
        assert lib().robe_cache_read(C.byref(c), P[6], 64, 4, 0, None) == BAD
    assert lib().robe_cache_write(C.byref(c), P[6], 64, 4, 0, None) == BAD


def test_cache_calls_refuse_their_rows():
    c = cache()
    for call in (lib().robe_cache_write, lib().robe_cache_read):
        for args in [(P[6], 64, 5, 0), (P[6], 63, 4, 0), (None, 64, 4, 0), (P[6], 64, -2, 0), (P[6], 64, 4, 2), (P[6], 64, 2**32 + 2, 0), (P[0], 64, 4, 0)]:
            assert call(C.byref(c), *args, None) == BAD, args
        assert call(None, P[6], 64, 4, 0, None) == BAD
        assert call(C.byref(c), None, 64, 0, 0, None) == robe.ROBE_OK
    none = cache(batch=0)
    assert lib().robe_cache_write(C.byref(none), P[6], 64, 4, 0, None) == BAD  # rows of no sequence at all, and nothing says which


def test_codes_and_scales_of_a_row_in_one_buffer_do_not_overlap():
    # rows of 64 codes and two scales, 72 bytes apart
    base = 0x10000
    c = cache(codes=C.c_void_p(base), codes_ld=72, codes_page=72 * 16, scales=C.c_void_p(base + 64), scales_ld=18, scales_page=18 * 16, num_pages=0)
    assert lib().robe_cache_write(C.byref(c), P[6], 64, 4, 0, None) == robe.ROBE_OK  # (no pages: checked, nothing launched)
    c = cache(codes=C.c_void_p(base), codes_ld=72, codes_page=72 * 16, scales=C.c_void_p(base + 60), scales_ld=18, scales_page=18 * 16)
    assert lib().robe_cache_write(C.byref(c), P[6], 64, 4, 0, None) == BAD


def attend(keys=None, values=None, **o):
    k = cache(group=32, starts=P[8], **(keys or {}))
    v = cache(group=32, starts=P[8], codes=P[3], scales=P[4], **(values or {}))
    a = dict(q=P[5], q_ld=32, q_seq=128, q_heads=4, bias=None, rows=None, rows_ld=4, out=P[6], out_ld=32, out_seq=128, ws=P[7], bytes=1 << 40)
    a.update(o)
    return lib().robe_cache_attention(C.byref(k), C.byref(v), a["q"], a["q_ld"], a["q_seq"], a["q_heads"], 1.0, a["bias"], a["rows"], a["rows_ld"], a["out"], a["out_ld"], a["out_seq"], a["ws"],
                                      a["bytes"], None)


@pytest.mark.parametrize("o", [dict(q=None), dict(out=None), dict(q_heads=3), dict(q_heads=0), dict(q_heads=2**20), dict(q_ld=31), dict(q_seq=127), dict(out_seq=0), dict(out_seq=-128), dict(out=P[5]), dict(out=P[0]), dict(out=P[7]),
                               dict(keys=dict(code_type=robe.ROBE_E4M3)), dict(values=dict(num_pages=9)), dict(values=dict(codes_ld=80, codes_page=80 * 16)), dict(values=dict(pages=P[9])),
                               dict(keys=dict(offsets=P[9]), values=dict(offsets=P[9])), dict(keys=dict(d=48), values=dict(d=48)), dict(keys=dict(codes=C.c_void_p(0x10008))),
                               dict(keys=dict(codes_ld=72, codes_page=72 * 16), values=dict(codes_ld=72, codes_page=72 * 16)),
                               dict(keys=dict(max_pages=2**28, pages_ld=2**28), values=dict(max_pages=2**28, pages_ld=2**28))])
def test_attention_refuses(o):
    assert attend(**o) == BAD


def test_attention_refuses_other_things():
    assert attend(ws=None) == WORK and attend(bytes=100) == WORK and attend(ws=C.c_void_p(0x7000010)) == WORK
    b = robe.robe_bias_create(8, 20, False)
    assert attend(bias=b) == BAD  # no rows
    assert attend(bias=b, rows=P[9], rows_ld=3) == BAD and attend(bias=b, rows=P[6]) == BAD
    robe.robe_bias_destroy(b)
    k = cache(group=32)  # no positions
    assert lib().robe_cache_attention(C.byref(k), C.byref(k), P[5], 32, 128, 4, 1.0, None, None, 0, P[6], 32, 128, P[7], 1 << 40, None) == BAD
    for dim in (16, 33, 48, 512):
        k = cache(d=2 * dim, group=dim, codes_ld=2 * dim, codes_page=32 * dim, starts=P[8])
        assert lib().robe_cache_attention(C.byref(k), C.byref(k), P[5], dim, 4 * dim, 4, 1.0, None, None, 0, P[6], dim, 4 * dim, P[7], 1 << 40, None) == BAD


def test_workspace_of_the_attention():
    need = robe.robe_cache_attention_workspace_bytes
    for bad in [(-1, 1, 1, 64, 10), (1, 0, 1, 64, 10), (1, 2, 3, 64, 10), (1, 1, 1, 48, 10), (1, 1, 1, 64, -1), (1, 1, 1, 64, 2**31), (2**31, 1, 1, 64, 10), (2**30, 2, 4, 64, 10),
                (2**70, 1, 1, 64, 10)]:
        assert need(*bad) == 0
    # spans are made for what is there, so a long page table asks for no more
    assert need(64, 8, 32, 128, 2**30) == need(64, 8, 32, 128, 2**20) < 16 << 20
    assert need(1, 1, 1, 32, 1) > 0


def test_binding_refuses_host_tensors_and_wrong_kinds():
    t, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        robe.robe_table_forward(t, ids, torch.zeros(3, 8))
    with pytest.raises(ValueError):
        robe.robe_table_backward(torch.zeros(3, 8), ids, t, None)
    with pytest.raises(ValueError):
        robe.robe_residual_quantize(t, None, None, torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1))
    codes, scales, pages = torch.zeros(2, 4, 8, dtype=torch.int8), torch.zeros(2, 4, 1), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        robe.robe_cache_write(t, codes, scales, pages)
    with pytest.raises(ValueError):
        robe.robe_cache_read(codes, scales, pages, t)
    with pytest.raises(ValueError):
        robe.robe_cache_attention(torch.zeros(1, 1, 32, dtype=torch.bfloat16), codes, scales, codes, scales, pages, torch.zeros(1, dtype=torch.int64), None, None, 1.0)
