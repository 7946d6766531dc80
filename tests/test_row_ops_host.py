"""Row operators without a GPU: the definitions against independent statements of them, the position buckets, argument
checks of the C ABI and of the binding."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2108_02191_b200 as robe
import rowops_reference as ref

BAD = robe.ROBE_ERR_INVALID_ARG
P = C.c_void_p(0x10000)   # never dereferenced
Q = C.c_void_p(0x4000000)
W = C.c_void_p(0x80000000)


def lib():
    return robe.binding.raw()


# ---------------------------------------------------------------- the definitions


def test_generator_known_answers():
    # published test vectors of Philox4x32-10: counter and key all zeros, all ones
    assert [int(v) for v in ref.philox(0, 0, 0, 0, 0)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 2**32 - 1
    assert [int(v) for v in ref.philox(ones, ones, ones, ones, 2**64 - 1)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_dropout_keeps_the_share_it_says():
    keep = ref.kept(500, 333, 0.3, 77, 5)
    n = keep.numel()
    q = 1 - ref.threshold(0.3) / 65536
    assert abs(float(keep.double().mean()) - q) < 5 * math.sqrt(q * (1 - q) / n)
    assert not torch.equal(keep, ref.kept(500, 333, 0.3, 77, 6))
    assert torch.equal(keep[:100, :64], ref.kept(100, 64, 0.3, 77, 5))  # a decision goes by its position alone


@pytest.mark.parametrize("two_sided", [False, True])
@pytest.mark.parametrize("buckets,far", [(2, 2), (4, 3), (32, 128), (32, 129), (6, 1000), (128, 65), (128, 2**30 - 1), (10, 12),
                                         (64, 100_000), (30, 128)])
def test_bucket_edges_are_exact(buckets, far, two_sided):
    if two_sided:
        buckets *= 2
    side = buckets // 2 if two_sided else buckets
    if far <= side // 2:
        pytest.skip("max_distance within the exact half")
    b = robe.robe_bias_create(buckets, far, two_sided)
    assert robe.robe_bias_num_buckets(b) == buckets
    edges = robe.robe_bias_get_edges(b)
    E = side // 2
    L = side - E
    assert edges[:E] == list(range(E)) and len(edges) == buckets
    for k in range(L):
        n, reach = edges[E + k], E ** (L - k) * far ** k
        assert n ** L >= reach > (n - 1) ** L
    if two_sided:
        assert edges[side:] == [max(1, v) for v in edges[:side]]
    # and the definition by distances, around every border
    for n in sorted({max(0, v + o) for v in edges[:side] for o in (-1, 0, 1)} | {far, far + 1, 2 * far}):
        want = max(k for k in range(side) if edges[k] <= n)
        assert ref.bucket(-n, buckets, far, two_sided) == want
    robe.robe_bias_destroy(b)


def test_usual_bucket_borders():
    # 32 two-sided buckets up to 128: 0..7 exact, then 8 sqrt(2)^k rounded up; the border at 16 = 8 sqrt(2)^2 is exact
    b = robe.robe_bias_create(32, 128, True)
    assert robe.robe_bias_get_edges(b)[:16] == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]
    robe.robe_bias_destroy(b)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate_rows", [None, "row", 1, 3])
def test_join_gradients_are_those_of_differences(layer, gate_rows):
    rows, d, eps = 6, 10, 1e-5
    rng = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=rng, dtype=torch.float64)
    factor = ref.kept(rows, d, 0.25, 9, 4).double() * ref.drop_scale(0.25)
    t = {"x": rnd(rows, d), "residual": rnd(rows, d), "w_post": rnd(d), "w_pre": rnd(d)}
    if gate_rows is not None:
        t["gate"] = rnd(rows, 1) if gate_rows == "row" else rnd(rows // gate_rows, d)
    go, gn = rnd(rows, d), rnd(rows, d)

    def loss(t):
        (out, _), (normed, _) = ref.join(t["x"], t["residual"], t["w_post"], t["w_pre"], t.get("gate"), 0.7, layer, eps, factor)
        return float((out * go).sum() + (normed * gn).sum())

    out = ref.join(t["x"], t["residual"], t["w_post"], t["w_pre"], t.get("gate"), 0.7, layer, eps, factor)[0][0]
    got = ref.join_grad(go, gn, t["x"], out, t["w_post"], t["w_pre"], t.get("gate"), 0.7, layer, eps, factor)
    h = 1e-5  # central differences: h^2 of the third derivative and 1e-16 / h of rounding, both below 1e-7 here
    for name, v in t.items():
        for k in range(0, v.numel(), 3):
            moved = []
            for sign in (1, -1):
                u = dict(t)
                u[name] = v.clone()
                u[name].reshape(-1)[k] += sign * h
                moved.append(loss(u))
            want = (moved[0] - moved[1]) / (2 * h)
            assert abs(float(got[name][0].reshape(-1)[k]) - want) < 1e-6 * (1 + abs(want)), (name, k)


# ---------------------------------------------------------------- argument checks of the C ABI


@pytest.mark.parametrize("args", [(1, 100, 0), (130, 1000, 0), (33, 100, 1), (2, 100, 1), (258, 1000, 1), (32, 16, 0), (32, 8, 1),
                                  (32, 2**30, 0), (32, 128, 2)])
def test_bias_create_refuses(args):
    b = robe.binding._BiasHandle()
    assert lib().robe_bias_create(C.byref(b), *args) == BAD and not b
    assert lib().robe_bias_create(None, 32, 128, 0) == BAD


def test_bias_handles_are_told_from_others():
    h = robe.robe_create(4096, 4, 16, 4, 7)
    as_bias = C.cast(h, robe.binding._BiasHandle)
    assert lib().robe_bias_num_buckets(as_bias) == BAD and lib().robe_bias_destroy(as_bias) == BAD
    assert lib().robe_bias_forward(as_bias, P, 4, 4, 1, 2, 2, 0, None, 0, Q, 2, 0, None) == BAD
    assert lib().robe_bias_num_buckets(None) == BAD and lib().robe_bias_destroy(None) == BAD
    assert lib().robe_bias_backward_workspace_bytes(as_bias, 4, 1, 2, 2) == 0
    with pytest.raises(C.ArgumentError):
        robe.robe_bias_num_buckets(h)
    robe.robe_destroy(h)


def test_bias_arguments():
    b = robe.robe_bias_create(32, 128, False)
    good = dict(rows=P, rows_ld=4, heads=4, batch=2, q=8, k=16, q_start=0, starts=None, causal=0, out=Q, ld=16, dtype=0)

    def forward(**change):
        a = dict(good, **change)
        return lib().robe_bias_forward(b, a["rows"], a["rows_ld"], a["heads"], a["batch"], a["q"], a["k"], a["q_start"], a["starts"],
                                       a["causal"], a["out"], a["ld"], a["dtype"], None)

    for change in (dict(rows=None), dict(rows=C.c_void_p(0x10002)), dict(rows_ld=3), dict(heads=0), dict(heads=1 << 22),
                   dict(batch=-1), dict(batch=1 << 31), dict(q=-1), dict(k=-1), dict(q=1 << 30, k=1 << 30), dict(causal=2),
                   dict(out=None), dict(out=C.c_void_p(0x4000001), dtype=1), dict(ld=15), dict(dtype=2),
                   dict(starts=C.c_void_p(0x80000004)), dict(out=P), dict(starts=Q), dict(ld=1 << 58)):
        assert forward(**change) == BAD, change
    assert forward(batch=0) == robe.ROBE_OK and forward(q=0) == robe.ROBE_OK and forward(k=0, out=None) == robe.ROBE_OK
    assert forward(batch=1 << 30, heads=1 << 20, rows_ld=1 << 20, q=1, k=1, ld=1, out=C.c_void_p(1 << 44)) == robe.ROBE_ERR_UNSUPPORTED  # 2^50 CTAs
    need = robe.robe_bias_backward_workspace_bytes(b, 4, 2, 8, 16)
    assert need > 0 and need % 256 == 0

    def backward(**change):
        a = dict(good, ws=W, ws_bytes=need, **{}) | change
        return lib().robe_bias_backward(b, a["out"], a["ld"], a["heads"], a["batch"], a["q"], a["k"], a["q_start"], a["starts"],
                                        a["causal"], a["dtype"], a["rows"], a["rows_ld"], a["ws"], a["ws_bytes"], None)

    for change in (dict(rows=None), dict(rows_ld=3), dict(out=None), dict(dtype=2), dict(causal=-1), dict(rows=Q), dict(heads=0)):
        assert backward(**change) == BAD, change
    for change in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=C.c_void_p(0x80000010))):
        assert backward(**change) == robe.ROBE_ERR_WORKSPACE, change
    assert backward(ws=C.c_void_p(0x10000)) == BAD  # the workspace over the result
    robe.robe_bias_destroy(b)


def test_bias_workspace_is_small():
    # a call's partial sums stay well below what it reads
    b = robe.robe_bias_create(32, 128, True)
    for n, h, q, k in [(16, 16, 2048, 2048), (1, 32, 4096, 4096), (4, 12, 777, 1001)]:
        assert robe.robe_bias_backward_workspace_bytes(b, h, n, q, k) < n * h * q * k * 2 / 32
    assert robe.robe_bias_backward_workspace_bytes(b, 4, 0, 8, 8) == 0
    robe.robe_bias_destroy(b)


def test_workspace_sizes_of_numbers_beyond_the_c_abis():
    b = robe.robe_bias_create(32, 128, True)
    for args in [(2**32 + 4, 1, 8, 8), (4, 2**64 + 1, 8, 8), (4, 1, 2**64 + 8, 8), (4, 1, 8, 2**64 + 8), (-4, 1, 8, 8)]:
        assert robe.robe_bias_backward_workspace_bytes(b, *args) == 0, args
    robe.robe_bias_destroy(b)
    for args in [(2**64 + 8, 16, 0), (8, 2**64 + 16, 0), (8, 16, 2**64 + 2), (8, 16, -1)]:
        assert robe.robe_residual_backward_workspace_bytes(*args) == 0, args


def test_dropout_arguments():
    def call(src=P, src_ld=10, out=Q, out_ld=10, rows=4, cols=10, dtype=0, p=0.1, step=None):
        return lib().robe_dropout(src, src_ld, out, out_ld, rows, cols, dtype, p, 1, 2, step, None)

    for change in (dict(src=None), dict(out=None), dict(src=C.c_void_p(0x10002)), dict(src_ld=9), dict(out_ld=9), dict(rows=-1),
                   dict(cols=-1), dict(rows=(1 << 32) + 1), dict(cols=(1 << 31) + 1), dict(dtype=2), dict(p=-0.1), dict(p=1.1),
                   dict(p=math.nan), dict(step=C.c_void_p(0x80000004)), dict(out=P, out_ld=12), dict(out=C.c_void_p(0x10004))):
        assert call(**change) == BAD, change
    assert call(rows=0, src=None, out=None) == robe.ROBE_OK and call(cols=0) == robe.ROBE_OK


def test_residual_arguments():
    S = robe.binding._Residual
    fields = dict(rows=8, d=16, dtype=0, norm=0, eps=1e-6, scale=1.0, gate=0, gate_rows=0, p=0.0, seed=1, offset=2, step=None)
    at = lambda k: C.c_void_p(0x100000 * k)

    def forward(spec=None, **change):
        c = S(*dict(fields, **(spec or {})).values())
        a = dict(x=at(1), x_ld=16, res=at(2), res_ld=16, gate=None, gate_ld=16, w1=at(4), w2=at(5), out=at(6), out_ld=16, n=at(7),
                 n_ld=16) | change
        return lib().robe_residual_forward(C.byref(c), *a.values(), None)

    for spec in (dict(rows=-1), dict(rows=(1 << 32) + 1), dict(d=0), dict(d=(1 << 20) + 1), dict(dtype=5), dict(norm=2),
                 dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(gate=3), dict(gate=2, gate_rows=3), dict(p=2.0),
                 dict(gate=2, gate_rows=0), dict(gate=1), dict(step=0x80000004)):
        assert forward(spec) == BAD, spec
    for change in (dict(x=None), dict(out=None), dict(n=None), dict(w2=None), dict(x_ld=15), dict(res_ld=15), dict(out_ld=15),
                   dict(n_ld=15), dict(gate=at(3)), dict(out=at(1)), dict(n=at(2)), dict(n=at(6)), dict(w1=C.c_void_p(0x400002)),
                   dict(out=at(2), out_ld=32), dict(n=at(5)), dict(out=C.c_void_p(0x200004))):
        assert forward(**change) == BAD, change
    assert forward(dict(gate=2, gate_rows=4), gate=at(3), gate_ld=15) == BAD
    assert forward(dict(rows=0), x=None, out=None, n=None, res=None) == robe.ROBE_OK
    assert lib().robe_residual_forward(None, *[None, 0] * 3, None, None, *[None, 0] * 2, None) == BAD

    need = robe.robe_residual_backward_workspace_bytes(8, 16, 0)
    assert need > 0 and need % 256 == 0

    def backward(spec=None, **change):
        c = S(*dict(fields, **(spec or {})).values())
        a = dict(go=at(1), go_ld=16, gn=at(2), gn_ld=16, x=at(3), x_ld=16, out=at(4), out_ld=16, gate=None, gate_ld=16, w1=at(6),
                 w2=at(7), gx=at(8), gx_ld=16, gr=at(9), gr_ld=16, gg=None, gg_ld=16, g1=at(11), g2=at(12), ws=at(13),
                 ws_bytes=need) | change
        return lib().robe_residual_backward(C.byref(c), *a.values(), None)

    for change in (dict(gn=None), dict(x=None), dict(out=None), dict(gx=None), dict(g1=None), dict(g2=None), dict(w1=None),
                   dict(w2=None), dict(gg=at(10)), dict(gx=at(1)), dict(gr=at(2)), dict(gr=at(1), gr_ld=32), dict(g1=at(12)),
                   dict(g1=at(6)), dict(gx=at(13)), dict(gx=at(9))):
        assert backward(**change) == BAD, change
    for change in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=C.c_void_p(0xD00010))):
        assert backward(**change) == robe.ROBE_ERR_WORKSPACE, change
    assert robe.robe_residual_backward_workspace_bytes(8, 16, 3) == 0
    assert robe.robe_residual_backward_workspace_bytes(-1, 16, 0) == 0


def test_a_step_counter_within_what_a_call_writes_is_refused():
    # every CTA reads the counter when it starts, others have written by then
    at = lambda k: C.c_void_p(0x100000 * k)
    assert lib().robe_dropout(at(1), 16, at(2), 16, 8, 16, 0, 0.1, 1, 2, 0x200000 + 504, None) == BAD
    assert lib().robe_dropout(at(1), 16, at(1), 16, 8, 16, 0, 0.1, 1, 2, 0x100000, None) == BAD  # in place too
    for step in (0x600000, 0x700008):  # out, normed
        c = robe.binding._Residual(8, 16, 0, 0, 1e-6, 1.0, 0, 0, 0.1, 1, 2, step)
        assert lib().robe_residual_forward(C.byref(c), at(1), 16, at(2), 16, None, 0, at(4), at(5), at(6), 16, at(7), 16, None) == BAD
    need = robe.robe_residual_backward_workspace_bytes(8, 16, 0)
    for step in (0x800000, 0x900100, 0xB00000, 0xC00038, 0xD00000 + need - 8):  # gradients of x, residual, both weights; workspace
        c = robe.binding._Residual(8, 16, 0, 0, 1e-6, 1.0, 0, 0, 0.1, 1, 2, step)
        assert lib().robe_residual_backward(C.byref(c), at(1), 16, at(2), 16, at(3), 16, at(4), 16, None, 0, at(6), at(7), at(8), 16,
                                            at(9), 16, None, 0, at(11), at(12), at(13), need, None) == BAD


@pytest.mark.parametrize("rows,d,gates", [(530_000, 4096, 0), (1 << 32, 300, 0), (1 << 32, 1 << 20, 0), (1 << 28, 512, 4), (1 << 28, 512, 1 << 19),
                                          (1 << 28, 512, 1 << 22), (1 << 30, 8, 0), (1 << 30, 8, 1 << 15), (1 << 30, 100, 1 << 29)])
def test_residual_sums_are_cut_so_that_no_thread_adds_up_many_rows(rows, d, gates):
    # the sums of every chunk are in the workspace, three of d fp32 each.  Rows of over 256 elements are one thread's after the
    # other; of shorter ones at least a 32nd of a chunk's
    chunks = robe.robe_residual_backward_workspace_bytes(rows, d, gates) // (12 * d)
    assert chunks * 256 * (1 if d > 256 else 32) >= rows
    assert chunks * 12 * d * 16 <= rows * d * 6  # and stay a small part of the call's tensors


def test_residual_beyond_a_grid():
    # the joining kernel would have 2^23 gate vectors of 2^12 CTAs each; (addresses are never reached)
    rows, d = 1 << 32, 1 << 20
    at = lambda k: C.c_void_p(k << 55)
    c = robe.binding._Residual(rows, d, 1, 0, 1e-6, 1.0, 2, 512, 0.0, 0, 0, None)
    need = robe.robe_residual_backward_workspace_bytes(rows, d, rows // 512)
    rc = lib().robe_residual_backward(C.byref(c), at(1), d, None, 0, at(2), d, None, 0, at(3), d, None, None, at(4), d, None, 0, at(5), d,
                                      None, None, at(6), need, None)
    assert rc == robe.ROBE_ERR_UNSUPPORTED


def test_column_slices_of_one_matrix_do_not_overlap():
    # rows of [8, 32]: the first 16 columns and the last 16; one column in common is refused
    c = robe.binding._Residual(8, 16, 0, 0, 1e-6, 1.0, 0, 0, 0.0, 1, 2, None)
    go = lambda out: lib().robe_residual_forward(C.byref(c), C.c_void_p(0x100000), 32, None, 0, None, 0, None, None,
                                                 C.c_void_p(out), 32, None, 0, None)
    assert go(0x100000 + 60) == BAD and go(0x100000 + 68) == BAD and go(0x100000 + 3 * 128 + 60) == BAD
    if not torch.cuda.is_available():  # a launch without a device is an error of its own, after all checks
        assert go(0x100000 + 64) == robe.ROBE_ERR_CUDA and go(0x100000 - 64) == robe.ROBE_ERR_CUDA


STUBS = r"""
#include <cuda_runtime.h>
#include <cstdio>
static cudaError_t told, left;  // what the helpers return, and the runtime's error that it leaves
static cudaError_t take_left() {
    const cudaError_t e = left;
    left = cudaSuccess;
    return e;
}
#define cudaGetLastError take_left
#include "robe_rows_api.cu"
namespace robe {
// launch helpers that fail as told, the runtime's error left set as by a call that only asks or sets something
cudaError_t fail() {
    left = told == kGridTooSmall ? cudaSuccess : told;
    return told;
}
cudaError_t launch_dropout(const void*, int64_t, void*, int64_t, int64_t, int64_t, int, const DropParams&, cudaStream_t) { return fail(); }
cudaError_t launch_bias_forward(const BiasProblem&, void*, int64_t, int, cudaStream_t) { return fail(); }
size_t bias_grad_workspace_bytes(uint32_t, uint32_t, int64_t, int64_t, int64_t) { return 0; }
cudaError_t launch_bias_backward(const BiasProblem&, const void*, int64_t, int, float*, int64_t, void*, cudaStream_t) { return fail(); }
cudaError_t launch_residual_forward(const ResidualProblem&, int, cudaStream_t) { return fail(); }
size_t residual_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }
cudaError_t launch_residual_backward(const ResidualProblem&, int, void*, cudaStream_t) { return fail(); }
}
int main() {
    char* p = (char*)0x100000;
    float* w = (float*)(p + 0x10000);
    robe_bias_t b;
    robe_bias_create(&b, 32, 128, 0);
    robe_residual_t c = {4, 8, ROBE_F32, 0, 1e-6f, 1.0f, 0, 0, 0.0f, 0, 0, nullptr};
    const cudaError_t all[] = {cudaErrorInvalidValue, cudaErrorInvalidConfiguration, kGridTooSmall};
    for (cudaError_t e : all) {
        told = e;
        for (int call = 0; call < 5; ++call) {
            const int rc = call == 0   ? robe_dropout(p, 8, p + 4096, 8, 4, 8, ROBE_F32, 0.1f, 1, 2, nullptr, nullptr)
                           : call == 1 ? robe_bias_forward(b, w, 4, 4, 1, 2, 8, 0, nullptr, 0, p, 8, ROBE_F32, nullptr)
                           : call == 2 ? robe_bias_backward(b, p, 8, 4, 1, 2, 8, 0, nullptr, 0, ROBE_F32, w, 4, nullptr, 0, nullptr)
                           : call == 3 ? robe_residual_forward(&c, p, 8, nullptr, 0, nullptr, 0, nullptr, nullptr, p + 4096, 8, nullptr, 0, nullptr)
                                       : robe_residual_backward(&c, p, 8, nullptr, 0, p + 4096, 8, nullptr, 0, nullptr, 0, nullptr, nullptr,
                                                                p + 8192, 8, nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr);
            printf("%d %d %d\n", (int)e, rc, (int)left);
        }
    }
}
"""


def test_errors_of_the_runtime_are_told_from_a_grids_limit_and_not_left_behind(tmp_path):
    # the C ABI's own source over launch helpers that fail: whatever the runtime answers is an error of its own, "unsupported"
    # only what a grid does not hold, and no error stays for the call after
    from paper_2108_02191_b200 import build
    src, exe = tmp_path / "status.cu", str(tmp_path / "status")
    src.write_text(STUBS)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, str(src)], check=True)
    lines = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")
    got = [tuple(int(v) for v in line.split()) for line in lines if line]
    assert len(got) == 15
    for told, status, left in got:
        assert status == (robe.ROBE_ERR_UNSUPPORTED if told == -1 else robe.ROBE_ERR_CUDA), (told, status)
        assert left == 0, (told, left)


# ---------------------------------------------------------------- the binding


def test_binding_refuses_host_tensors_and_wrong_kinds():
    x = torch.zeros(4, 8)
    b = robe.robe_bias_create(32, 128, False)
    for call in (lambda: robe.robe_dropout(x, x, 0.1, 1), lambda: robe.robe_bias_forward(b, x, x[None], 0),
                 lambda: robe.robe_bias_backward(b, x[None], x, None, 0), lambda: robe.robe_residual_forward(x, None, x),
                 lambda: robe.robe_residual_backward(x, None, x, None, x)):
        with pytest.raises(ValueError):
            call()
    robe.robe_bias_destroy(b)
