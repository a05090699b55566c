"""The 4-bit cache's layout and page arithmetic (csrc/q4_format.h, compiled on
its own), its quantiser's rounding, and the calls' refusals, on the CPU."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import q4_oracle as Q
from paper_2607_13205_gb300 import build as B
from paper_2607_13205_gb300 import rolekv as R

SHIM = r"""
#include "q4_format.h"
using namespace rolekv;
extern "C" {
int k_piece(int d, int row, int e) { return q4_k_piece(d, row, e); }
int v_piece(int d, int row, int e) { return q4_v_piece(d, row, e); }
int scale_at(int d, int row, int j) { return q4_scale(d, row, j); }
int k_scales(int d) { return q4_k_scales(d); }
int v_scales(int d) { return q4_v_scales(d); }
unsigned quotient(unsigned n, unsigned d) { return n / make_div(d); }
int clamp_rows(long len, long cap) { return q4_clamp_rows(len, cap); }
long record(const int* row, int max_pages, int n_pages, int recs, long sl, long sp, int d, int l, int h, int rec) {
  return q4_record_at(row, max_pages, n_pages, make_div(recs), sl, sp, d, l, h, rec);
}
}
"""


@pytest.fixture(scope="module")
def fmt(tmp_path_factory):
    d = tmp_path_factory.mktemp("q4")
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", B.CSRC, "-o", so, src], check=True)
    lib = ctypes.CDLL(so)
    L, I = ctypes.c_long, ctypes.c_int
    lib.record.argtypes = [ctypes.POINTER(I), I, I, I, L, L, I, I, I, I]
    lib.record.restype = L
    lib.clamp_rows.argtypes = [L, L]
    return lib


@pytest.mark.parametrize("d", [64, 128])
def test_every_byte_of_a_record_belongs_to_one_row(fmt, d):
    """Pieces and scales of the 16 rows tile the record, and hold what the
    oracle's element-by-element layout says."""
    owner = {}
    for row in range(16):
        for e in range(0, d, 4):
            for at in (fmt.k_piece(d, row, e), fmt.v_piece(d, row, e)):
                assert at % 2 == 0
                for x in (at, at + 1):
                    assert owner.setdefault(x, (row, e, at)) == (row, e, at)
        for j in range(d // 32):
            for s0 in (fmt.k_scales(d), fmt.v_scales(d)):
                for x in (0, 1):
                    assert owner.setdefault(s0 + fmt.scale_at(d, row, j) + x, (row, j, s0)) == (row, j, s0)
    assert sorted(owner) == list(range(18 * d))
    rng = np.random.default_rng(d)
    k, v = (torch.randn(16, d, generator=torch.Generator().manual_seed(i)).bfloat16().double().numpy() for i in (1, 2))
    rec = rng.integers(0, 256, 18 * d).astype(np.uint8)
    for row in range(16):
        Q.write_row(rec, row, k[row], v[row])
    for row in range(16):
        for x, piece, s0 in ((k, fmt.k_piece, fmt.k_scales(d)), (v, fmt.v_piece, fmt.v_scales(d))):
            code, s = Q.quantise(x[row])
            for e in range(d):
                at = piece(d, row, e - e % 4)
                word = int(rec[at]) | (int(rec[at + 1]) << 8)
                assert (word >> (4 * (e % 4))) & 15 == code[e] + 8
            for j in range(d // 32):
                at = s0 + fmt.scale_at(d, row, j)
                assert int(rec[at]) | (int(rec[at + 1]) << 8) == Q.scale_bits(s)[j]
        got = Q.read_row(rec, row)
        assert np.array_equal(got[0], Q.values(k[row])) and np.array_equal(got[1], Q.values(v[row])) and not got[2]


def test_bad_pages_have_no_record(fmt):
    row = (ctypes.c_int * 3)(4, -1, 9)
    args = (3, 9, 2, 1 << 40, 5 * 2 * 2304, 128)
    page, head = 5 * 2 * 2304, 2 * 2304
    assert fmt.record(row, *args, 0, 0, 0) == 4 * page
    assert fmt.record(row, *args, 3, 2, 1) == 3 * (1 << 40) + 4 * page + 2 * head + 2304   # (past 32 bits)
    assert fmt.record(row, *args, 0, 0, 2) == -1        # no page there
    assert fmt.record(row, *args, 0, 0, 4) == -1        # a page past the pool
    assert fmt.record(row, *args, 0, 0, 6) == -1        # past the table
    assert fmt.record(row, *args, 0, 0, -1) == -1
    assert fmt.record(row, 3, 10, 2, 0, page, 128, 0, 0, 4) == 9 * page
    assert [fmt.clamp_rows(x, 96) for x in (-5, 0, 96, 97, 1 << 40)] == [0, 0, 96, 96, 96]


def test_division_by_a_product(fmt):
    fmt.quotient.restype = ctypes.c_uint
    fmt.quotient.argtypes = [ctypes.c_uint] * 2
    rng = np.random.default_rng(0)
    top = 2 ** 31 - 1
    ds = [1, 2, 3, 4, 5, 7, 63, 64, 65, 641, 4095, 4096, 65537, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, top] + \
        [int(x) for x in rng.integers(1, top, 200)]
    for d in ds:
        q = top // d
        for n in {0, 1, d - 1, d, top, top - 1, q * d, max(0, q * d - 1)} | {int(x) for x in rng.integers(0, top, 20)}:
            assert fmt.quotient(n, d) == n // d, (n, d)


def test_code_rounding_over_all_mantissas():
    """floor(x / s + 1/2) from one fused multiply-add and one addition: for
    every pair of 8-bit mantissas and every exponent that gives |x / s| <=
    7 (1 + 2^-8) (s is m / 7 to eight bits) the fp32 steps agree with the exact quotient, half-way ones included."""
    a, b = np.meshgrid(np.arange(128, 256), np.arange(128, 256), indexing="ij")
    ties = 0
    for k in range(-12, 4):
        for sign in (1, -1):
            x = sign * np.ldexp(a.astype(np.float64), k)
            s = b.astype(np.float64)
            ok = np.abs(x) <= 7.0 * (1 + 2.0 ** -8) * s
            inv = (np.float32(1) / s.astype(np.float32)).astype(np.float64)
            t = (x * inv + (8.0 + 2.0 ** -14)).astype(np.float32)       # (exact in fp64, one rounding: the fma)
            n = (t + np.float32(8388608.0)).view(np.uint32) & 15
            num = (2 * sign * a * 2 ** (k + 12) + b * 2 ** 12)          # 2^12 (2 x + s) over 2^13 s, whole numbers
            want = num // (b * 2 ** 13) + 8
            assert np.array_equal(n[ok], want[ok])
            ties += int((num[ok] % (b * 2 ** 13)[ok] == 0).sum())
    assert ties > 100


def test_scale_rounding_over_all_mantissas():
    """m / 7 rounded to fp32 and then to bf16 is the exact quotient to bf16."""
    m = np.arange(128, 256, dtype=np.float64)
    q32 = (m.astype(np.float32) / np.float32(7)).view(np.uint32)
    twice = ((q32 + 0x7FFF + ((q32 >> 16) & 1)) >> 16).astype(np.uint16)
    _, s = Q.quantise(np.repeat(m[:, None], 32, 1))
    assert np.array_equal(twice, Q.scale_bits(s[:, 0]))


# ------------------------------------------------------------------ refusals ----

@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        B.build()
    return R.lib()


def _pages(**kw):
    a = dict(n_seqs=4, max_pages=8, n_pages=20, page_rows=32, table=256, lens=256, refs=256)
    a.update(kw)
    return R.PagesDesc(*a.values())


def _pool(**kw):
    a = dict(ptr=256, L=2, Hkv=2, d=128, s_layer=20 * 2 * 2 * 2304, s_page=2 * 2 * 2304)
    a.update(kw)
    return R.PoolDesc(*a.values())


def _ref(x):
    return None if x is None else ctypes.byref(x)


FAKE = ctypes.c_void_p(256)            # never dereferenced: the checks fail first
BIG = 1 << 30


def _calls(lib, pages, pool, b=4, ptr=FAKE, ws=FAKE, ws_bytes=BIG):
    """Every call of the paged cache with these tables."""
    t = R.Tensor(256, 1 << 20, 1 << 16, 1 << 10, 128)
    batch = R.BatchDesc(2, b, 4, 2, 128, 100, None, None)
    return {
        "reserve": lambda: lib.kv_pages_reserve(_ref(pages), _ref(pool), ptr, ptr, ws, ws_bytes, None, None),
        "fork": lambda: lib.kv_pages_fork(_ref(pages), ptr, ws, ws_bytes, None, None),
        "pack": lambda: lib.kv_pages_pack(_ref(pages), _ref(pool), None, ws, ws_bytes, None, None),
        "compact": lambda: lib.kv_compact_q4(ctypes.byref(batch), t, t, ptr, 0.5, _ref(pool), _ref(pages), None, ptr,
                                             None, None),
        "append": lambda: lib.kv_append_q4(_ref(pool), _ref(pages), None, b, t, t, 1, None, ptr, None, None),
        "expand": lambda: lib.kv_expand_q4(_ref(pool), _ref(pages), None, b, None, 4, t, t, None, None),
        "decode": lambda: lib.decode_attention_q4(_ref(pool), _ref(pages), None, b, 4, t, 0.0, ptr, ws, ws_bytes,
                                                  None, None),
    }


ALL = ["reserve", "fork", "pack", "compact", "append", "expand", "decode"]
POOLED = [c for c in ALL if c != "fork"]
INV, UNS, WS = R.ERR_INVALID_ARG, R.ERR_UNSUPPORTED, R.ERR_WORKSPACE


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("change, code", [
    (dict(n_seqs=0), INV), (dict(max_pages=0), INV), (dict(n_pages=0), INV), (dict(table=None), INV),
    (dict(lens=None), INV), (dict(refs=None), INV), (dict(table=258), INV), (dict(page_rows=24), UNS),
    (dict(page_rows=0), UNS), (dict(page_rows=8192), UNS), (dict(max_pages=1 << 28), UNS)])
def test_bad_tables_are_refused(lib, call, change, code):
    assert _calls(lib, _pages(**change), _pool())[call]() == code
    assert lib.rolekv_last_error()


@pytest.mark.parametrize("call", POOLED)
@pytest.mark.parametrize("change, code", [
    (dict(ptr=None), INV), (dict(ptr=264), INV), (dict(L=0), INV), (dict(Hkv=0), INV), (dict(d=96), UNS),
    (dict(s_page=2 * 2 * 2304 - 16), INV), (dict(s_page=2 * 2 * 2304 + 8), INV), (dict(s_layer=-16), INV),
    (dict(s_layer=16), INV)])
def test_bad_pools_are_refused(lib, call, change, code):
    assert _calls(lib, _pages(), _pool(**change))[call]() == code


@pytest.mark.parametrize("call", ALL)
def test_missing_arguments_are_refused(lib, call):
    assert _calls(lib, None, _pool())[call]() == INV
    if call in POOLED:
        assert _calls(lib, _pages(), None)[call]() == INV
    if call not in ("pack", "expand"):
        assert _calls(lib, _pages(), _pool(), ptr=None)[call]() == INV
        assert _calls(lib, _pages(), _pool(), ptr=ctypes.c_void_p(258))[call]() == INV
    if call in ("compact", "append", "expand", "decode"):
        assert _calls(lib, _pages(), _pool(), b=5)[call]() == INV       # more sequences than slots
    if call in ("reserve", "fork", "pack", "decode"):
        assert _calls(lib, _pages(), _pool(), ws=None)[call]() == WS
        assert _calls(lib, _pages(), _pool(), ws_bytes=16)[call]() == WS
        assert _calls(lib, _pages(), _pool(), ws=ctypes.c_void_p(264))[call]() == WS


def test_batch_and_pool_agree(lib):
    t = R.Tensor(256, 1 << 20, 1 << 16, 1 << 10, 128)
    for change in (dict(L=3), dict(Hkv=1, Hq=1), dict(d=64)):
        a = dict(L=2, b=4, Hq=4, Hkv=2, d=128)
        a.update(change)
        batch = R.BatchDesc(*a.values(), 100, None, None)
        assert lib.kv_compact_q4(ctypes.byref(batch), t, t, FAKE, 0.5, _ref(_pool()), _ref(_pages()), None, FAKE, None,
                                 None) == INV
    batch = R.BatchDesc(2, 4, 4, 2, 128, 100, None, None)
    for budget in (0.0, 1.5, float("nan")):
        assert lib.kv_compact_q4(ctypes.byref(batch), t, t, FAKE, budget, _ref(_pool()), _ref(_pages()), None, FAKE,
                                 None, None) == INV
    bad = R.Tensor(256, 1 << 20, 1 << 16, 1 << 10, 132)
    for k, v in ((bad, t), (t, bad)):
        assert lib.kv_append_q4(_ref(_pool()), _ref(_pages()), None, 4, k, v, 1, None, FAKE, None, None) == INV
        assert lib.kv_expand_q4(_ref(_pool()), _ref(_pages()), None, 4, None, 4, k, v, None, None) == INV
    assert lib.kv_append_q4(_ref(_pool()), _ref(_pages()), None, 4, t, t, -1, None, FAKE, None, None) == INV
    assert lib.kv_expand_q4(_ref(_pool()), _ref(_pages()), None, 4, None, -1, t, t, None, None) == INV


def test_decode_refusals(lib):
    t = R.Tensor(256, 1 << 20, 1 << 16, 1 << 10, 128)

    def go(Hq=4, q=t, b=4, out=FAKE):
        return lib.decode_attention_q4(_ref(_pool()), _ref(_pages(n_seqs=8192)), None, b, Hq, q, 0.0, out, FAKE, BIG,
                                       None, None)
    assert go(Hq=3) == INV and go(Hq=0) == INV
    assert go(Hq=18) == UNS
    assert go(b=4097) == UNS and go(b=0) == INV
    assert go(q=R.Tensor(264, 1 << 20, 1 << 16, 1 << 10, 128)) == INV
    assert go(q=R.Tensor(256, 1 << 20, 1 << 16, 100, 128)) == INV
    assert go(out=None) == INV and go(out=ctypes.c_void_p(264)) == INV


def test_sizes(lib):
    assert lib.rolekv_q4_page_bytes(8, 128, 64) == 8 * 4 * 18 * 128
    for bad in ((0, 128, 64), (8, 96, 64), (8, 128, 8), (8, 128, 40), (8, 128, 8192)):
        assert lib.rolekv_q4_page_bytes(*bad) == -1
    out = ctypes.c_size_t(0)
    assert lib.rolekv_pages_workspace_size(_ref(_pages()), None) == INV
    assert lib.rolekv_pages_workspace_size(_ref(_pages(page_rows=8)), ctypes.byref(out)) == UNS
    assert lib.rolekv_pages_workspace_size(_ref(_pages()), ctypes.byref(out)) == 0
    assert out.value >= 4 * max(4 * 9, 3 * 20)
    assert lib.rolekv_decode_q4_workspace_size(1, 1, 8, 2, 64, None) == INV
    assert lib.rolekv_decode_q4_workspace_size(1, 1, 7, 2, 64, ctypes.byref(out)) == INV
    assert lib.rolekv_decode_q4_workspace_size(1, 1, 8, 2, 64, ctypes.byref(out)) == 0 and out.value > 0


def test_binding_checks():
    """What the binding refuses before the library is asked."""
    pages = R.Pages(2, 5, 32, 4, device="cpu")
    assert pages.state.numel() == 2 * 4 + 2 + 5 and (pages.table == -1).all()
    pool = torch.zeros(R.q4_pool_shape(1, 5, 2, 64, 32), dtype=torch.uint8)
    assert pool.shape == (1, 5, 2, 2, 18 * 64)
    d = R.pool_desc(pool, pages)
    assert (d.L, d.Hkv, d.d, d.s_page) == (1, 2, 64, 2 * 2 * 18 * 64)
    with pytest.raises(ValueError):
        R.q4_pool_shape(1, 5, 2, 96, 32)
    with pytest.raises(TypeError):
        R.pool_desc(pool.int(), pages)
    with pytest.raises(ValueError):
        R.pool_desc(pool[:, :4], pages)
    with pytest.raises(ValueError):
        R.pool_desc(torch.zeros((1, 5, 2, 4, 18 * 64), dtype=torch.uint8)[:, :, :, ::2], pages)
    for bad in (torch.zeros(3, dtype=torch.int32), torch.zeros(2), torch.zeros((2, 2), dtype=torch.int32)[:, 0]):
        with pytest.raises(ValueError):
            R._int32(bad, 2, "pos")


def test_binding_checks_the_batch():
    """Sizes that the library cannot see: k, v and keep_idx of another batch."""
    batch = R.Batch(1, 2, 2, 2, 64, 10, device="cpu")
    assert batch.kept_total(0.35) == 2 * R.kept_rows(10, 0.35) and batch.kept_total(0.35) == 8
    ragged = R.Batch(1, 3, 2, 2, 64, 10, seqlens=[10, 0, 3], device="cpu")
    assert ragged.kept_total(0.5) == 5 + 0 + 2


def test_expand_refuses_shared_outputs(lib):
    t = R.Tensor(256, 1 << 20, 1 << 16, 1 << 10, 128)
    for bad in (R.Tensor(256, 0, 1 << 16, 1 << 10, 128), R.Tensor(256, 1 << 20, 0, 1 << 10, 128),
                R.Tensor(256, 1 << 20, 1 << 16, 0, 128)):
        for k, v in ((bad, t), (t, bad)):
            assert lib.kv_expand_q4(_ref(_pool()), _ref(_pages()), None, 4, None, 4, k, v, None, None) == INV


def test_reserve_refuses_overlapping_arrays(lib):
    """The kernel reads add and the lengths again after pos is written."""
    pages, pool = _pages(table=1 << 20, lens=1 << 21, refs=1 << 22), _pool()
    at = [1 << 24, (1 << 24) + 12, 1 << 21, (1 << 21) - 12, (1 << 22) + 76, (1 << 20) + 4 * 31]
    for x in range(len(at)):
        for y in range(len(at)):
            if x < 2 and y < 2 or min(x, y) == 0 and max(x, y) in (2, 3):
                got = lib.kv_pages_reserve(_ref(pages), _ref(pool), ctypes.c_void_p(at[x]), ctypes.c_void_p(at[y]),
                                           FAKE, BIG, None, None)
                assert got == INV, (x, y)
    for y in at[2:]:
        assert lib.kv_pages_reserve(_ref(pages), _ref(pool), ctypes.c_void_p(1 << 24), ctypes.c_void_p(y), FAKE, BIG,
                                    None, None) == INV


def test_decode_refuses_more_rows_than_it_counts(lib):
    """Pieces of 32 rows are counted in 32 bits."""
    def go(b, **kw):
        pages = _pages(n_seqs=b, page_rows=4096, max_pages=(1 << 18) - 1, n_pages=4)
        kw = dict(dict(L=1, Hkv=1), **kw)
        page = kw["Hkv"] * 256 * 2304
        pool = _pool(s_page=page, s_layer=4 * page, **kw)
        q = R.Tensor(256, 0, 0, 128, 0)
        return lib.decode_attention_q4(_ref(pool), _ref(pages), None, b, kw["Hkv"], q, 0.0, FAKE, None, 0, None, None)
    assert go(64) == WS                       # (2^31 - 2^13 pieces: the next check, of the workspace, fails)
    assert go(65) == UNS
    assert go(64, Hkv=60000) == UNS           # (more of them than 2^31 a CTA)


def test_books_of_many_slots_are_taken(lib):
    """Slots times layers and heads are no batch: the next check, of the
    workspace, is the one that fails."""
    pages, pool = _pages(n_seqs=20000), _pool(L=32, Hkv=8, s_page=8 * 2 * 2304, s_layer=20 * 8 * 2 * 2304)
    for call in ("reserve", "pack"):
        assert _calls(lib, pages, pool, ws=None, ws_bytes=0)[call]() == WS
    assert _calls(lib, pages, pool, b=20000)["append"]() == UNS         # (that is one)


def test_calls_refuse_arrays_that_are_their_tables(lib):
    """add, parent and n_live inside an array that the call writes."""
    pages, pool = _pages(table=1 << 20, lens=1 << 21, refs=1 << 22), _pool()
    p = ctypes.c_void_p
    for at in (1 << 20, (1 << 20) + 4 * 31, (1 << 20) - 12, 1 << 21, (1 << 21) + 12, 1 << 22, (1 << 22) + 76):
        assert lib.kv_pages_reserve(_ref(pages), _ref(pool), p(at), p(1 << 24), FAKE, BIG, None, None) == INV, hex(at)
        assert lib.kv_pages_fork(_ref(pages), p(at), FAKE, BIG, None, None) == INV, hex(at)
    for at in (1 << 20, (1 << 20) + 4 * 31, 1 << 21, (1 << 21) + 12, 1 << 22, (1 << 22) + 76):
        assert lib.kv_pages_pack(_ref(pages), _ref(pool), p(at), FAKE, BIG, None, None) == INV, hex(at)


def test_rows_written_at_once():
    """The oracle's two ways to write rows are the same."""
    for d in (64, 128):
        rng = np.random.default_rng(d)
        g = torch.Generator().manual_seed(d)
        k, v = (torch.randn(40, d, generator=g).bfloat16().double().numpy() for _ in "kv")
        k[3, 5], v[4, 40] = np.inf, np.nan
        place = rng.permutation(5 * 16)[:40]
        empty = rng.random(40) < 0.2
        want = rng.integers(0, 256, (5, 18 * d)).astype(np.uint8)
        got = want.copy()
        for i in range(40):
            Q.write_row(want[place[i] // 16], int(place[i] % 16), k[i], v[i], bool(empty[i]))
        Q.write_rows(got, place // 16, place % 16, k, v, empty)
        assert np.array_equal(got, want)


def _bf16(x32):
    """fp32 to bf16 bits, ties to even."""
    u = x32.view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def test_scale_by_a_product_over_all_maxima():
    """The kernels take m / 7 as a product with fp32's 1/7, rounded to fp32 and
    then to bf16, and 0 where that is below 2^-126: the exact quotient's scale for
    every finite bf16 m."""
    m = (np.arange(0x7F80, dtype=np.uint32) << 16).view(np.float32)
    bits = _bf16(m * (np.float32(1) / np.float32(7)))
    bits[bits < 0x0080] = 0
    _, s = Q.quantise(np.repeat(m.astype(np.float64)[:, None], 32, 1))
    assert np.array_equal(bits, Q.scale_bits(s[:, 0]))


@pytest.mark.parametrize("off", [-1, 0, 1])
@pytest.mark.parametrize("form", ["nibble", "byte"])
def test_codes_with_an_approximate_reciprocal(form, off):
    """Both of the kernels' forms of floor(x / s + 1/2) + 8, one fused
    multiply-add each, with a reciprocal that is one unit in the last place off
    (as much as the approximate instruction may be): the exact quotient's code
    for every pair of 8-bit mantissas, ties among them."""
    a, b = np.meshgrid(np.arange(128, 256), np.arange(128, 256), indexing="ij")
    ties = 0
    s32 = b.astype(np.float32)
    inv = ((np.float32(1) / s32).view(np.uint32) + np.uint32(off & 0xFFFFFFFF)).view(np.float32).astype(np.float64)
    for k in range(-12, 4):
        for sign in (1, -1):
            x = sign * np.ldexp(a.astype(np.float64), k)
            ok = np.abs(x) <= 7.0 * (1 + 2.0 ** -8) * b
            if form == "nibble":
                t = (x * inv + (8.0 + 2.0 ** -14)).astype(np.float32)          # (exact in fp64, one rounding: the fma)
                n = (t + np.float32(8388608.0)).view(np.uint32) & 15
            else:
                t = (x * inv + (136.5 + 2.0 ** -14)).astype(np.float32)
                n = (t.view(np.uint32) >> 16) & 255
            num = 2 * sign * a * 2 ** (k + 12) + b * 2 ** 12        # 2^12 (2 x + s) over 2^13 s, whole numbers
            want = num // (b * 2 ** 13) + 8
            assert np.array_equal(n[ok], want[ok])
            ties += int((num[ok] % (b * 2 ** 13)[ok] == 0).sum())
    assert ties > 100
