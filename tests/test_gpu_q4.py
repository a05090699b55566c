"""The paged 4-bit cache on the GPU against the fp64 oracle: rows stored are
the oracle's bytes, rows read back its values, the book its lists, and
attention its sums."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import q4_oracle as Q
from paper_2607_13205_gb300 import inputs as I
from paper_2607_13205_gb300 import rolekv as R
from tests.q4_helpers import DEV, Cache, bf16, check_attention, f64, i32

pytestmark = pytest.mark.gpu


def new_status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def pages_for(lens, P, extra=3):
    return sum(-(-n // P) for n in lens) + extra


# --------------------------------------------------------------- rows stored ----

@pytest.mark.parametrize("d, P, T, base", [(128, 16, 1, 0), (128, 64, 1, 63), (64, 32, 1, 31), (128, 48, 3, 46),
                                           (64, 16, 40, 5), (128, 32, 70, 16)])
def test_append_writes_the_oracles_bytes(d, P, T, base):
    """New rows of every sequence (one gets none, one fewer); nothing else in
    the pool changes."""
    L, Hkv, b = 2, 3, 4
    lens = [base + T] * b
    c = Cache(b, pages_for(lens, P), P, -(-(base + T) // P) + 1, L, Hkv, d, seed=T).fill(lens, shuffle=1)
    k, v = bf16((L, b, Hkv, T, d), 1), bf16((L, b, Hkv, T, d), 2, 3.0)
    pos, count = [base, -1, base, base], [T, T, T - 1, T + 5]
    for s in range(b):
        for i in range(0 if pos[s] < 0 else min(T, count[s])):
            for l in range(L):
                for h in range(Hkv):
                    c.write(s, l, h, base + i, f64(k[l, s, h, i]), f64(v[l, s, h, i]))
    st = new_status()
    R.kv_append_q4(c.pool, c.pages, k.to(DEV), v.to(DEV), i32(pos), count=i32(count), status=st)
    c.check_pool()
    assert st.item() == 0


def special_rows(d):
    """Rows of bf16 values at which the quantiser could go wrong."""
    x = torch.zeros(14, d)
    g = torch.Generator().manual_seed(3)
    x[1] = torch.randn(d, generator=g)
    x[1, :32] = 0                                            # a zero group beside others
    x[2] = 2.0 ** -133                                       # bf16's least: scale below 2^-126
    x[3] = torch.randn(d, generator=g) * 2.0 ** -123         # about 2^-126 for the scale
    x[4] = 3.3e38 * torch.sign(torch.randn(d, generator=g))  # bf16's largest
    x[5] = 7.0 * torch.arange(d).remainder(3).sub(1)
    x[6] = torch.arange(d).remainder(15).sub(7).float()      # scale 1: whole codes
    x[7] = torch.arange(d).remainder(29).sub(14).float() / 2 # scale 1: half-way codes
    x[8] = 1.75 * torch.arange(d).remainder(29).sub(14).float() / 2 / 1.75
    x[9] = torch.randn(d, generator=g)
    x[9, 40] = float("inf")
    x[10] = torch.randn(d, generator=g)
    x[10, 3] = float("nan")
    x[11] = -torch.rand(d, generator=g)
    x[12] = torch.exp(torch.randn(d, generator=g) * 10)
    x[13, 33] = -2.0 ** -126 * 7
    return x.bfloat16()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("through", ["append", "compact"])
def test_special_values(d, through):
    x = special_rows(d)
    n = x.shape[0]
    k, v = x, x.flip(0)
    c = Cache(1, 3, 16, 2, 1, 1, d, seed=5).fill([n], shuffle=2)
    for r in range(n):
        c.write(0, 0, 0, r, f64(k[r]), f64(v[r]))
    st = new_status()
    kd, vd = k.to(DEV).view(1, 1, 1, n, d), v.to(DEV).view(1, 1, 1, n, d)
    if through == "append":
        R.kv_append_q4(c.pool, c.pages, kd, vd, i32([0]), status=st)
    else:
        batch = R.Batch(1, 1, 1, 1, d, n)
        R.kv_compact_q4(batch, kd, vd, i32(list(range(n))).view(1, 1, 1, n), 1.0, c.pool, c.pages, i32([0]), status=st)
    c.check_pool()
    assert st.item() == R.STATUS_NONFINITE
    out = [torch.zeros((1, 1, 1, n, d), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    R.kv_expand_q4(c.pool, c.pages, *out)
    rows = c.rows(0, 0, 0)
    for o, want in zip(out, rows):
        assert torch.equal(torch.nan_to_num(o[0, 0, 0].cpu(), nan=-5.0),
                           torch.nan_to_num(torch.from_numpy(want).float().bfloat16(), nan=-5.0))


@pytest.mark.parametrize("d, P, lens, budget, base, packed, extra", [
    (128, 64, [700, 700], 0.3, 0, False, 0),
    (64, 16, [333, 333, 333], 0.11, 7, False, 0),
    (128, 48, [130, 0, 1, 517, 64], 0.25, 0, True, 0),
    (64, 32, [90, 5, 300], 0.5, 17, True, 2),
    (128, 128, [1000], 1.0, 1, False, 0),
    (128, 16, [40, 40], 0.02, 15, False, 0)])
def test_compact_writes_the_oracles_bytes(d, P, lens, budget, base, packed, extra):
    """Kept rows behind `base` earlier ones, slots without a token among them;
    rows before and behind, and the other pages, stay as they were."""
    L, Hkv, b = 2, 2, len(lens)
    kept = [R.kept_rows(n, budget, extra) for n in lens]
    rows = [base + m for m in kept]
    c = Cache(b, pages_for(rows, P), P, -(-max(rows) // P) + 1, L, Hkv, d, seed=1).fill(rows, shuffle=3)
    rng = np.random.default_rng(len(lens))
    idx = [np.stack([np.stack([np.sort(rng.choice(n, m, replace=False)) for _ in range(Hkv)]) for _ in range(L)])
           if m else np.zeros((L, Hkv, 0), np.int64) for n, m in zip(lens, kept)]
    for s, m in enumerate(kept):
        if m > 3:
            idx[s][:, :, m - 2:] = -1
            idx[s][0, 1, m // 2] = -1                         # (and one in the middle of one head's)
    batch = R.Batch(L, b, Hkv, Hkv, d, max(lens), seqlens=lens if packed else None, kept_extra=extra)
    if packed:
        T = sum(lens)
        k, v = bf16((L, T, Hkv, d), 1), bf16((L, T, Hkv, d), 2)
        at = np.cumsum([0] + lens)
        src = [lambda x, l, s, h, t: x[l, at[s] + t, h]] * 2
        keep = np.concatenate(idx, -1)
    else:
        # heads inside the token rows, as a projection leaves them
        k, v = (bf16((L, b, lens[0], Hkv, d), x).transpose(2, 3) for x in (1, 2))
        src = [lambda x, l, s, h, t: x[l, s, h, t]] * 2
        keep = np.stack(idx, 1)
    for s, m in enumerate(kept):
        for l in range(L):
            for h in range(Hkv):
                for j in range(m):
                    t = int(idx[s][l, h, j])
                    kk, vv = (f64(src[0](x, l, s, h, max(t, 0))) for x in (k, v))
                    c.write(s, l, h, base + j, kk, vv, empty=t < 0)
    st = new_status()
    kd, vd = k.to(DEV), v.to(DEV)
    R.kv_compact_q4(batch, kd, vd, i32(keep.tolist()), budget, c.pool, c.pages, i32([base] * b), status=st)
    c.check_pool()
    assert st.item() == 0


def test_compact_into_chosen_slots():
    """A batch of two prompts into slots 5 and 2; a slot named twice is written
    once; one out of range, one without room and an index past the end of its
    sequence are reported and skipped."""
    d, P, L, Hkv, n = 128, 16, 1, 2, 40
    def fresh():
        c = Cache(6, 20, P, 4, L, Hkv, d, seed=2)
        c.book.lens[:] = [0, 0, 10, 0, 0, 10]
        for s, pg in ((2, 7), (5, 3)):
            c.book.table[s][0] = pg
            c.book.refs[pg] = 1
        c.upload()
        return c
    k, v = bf16((L, 3, Hkv, n, d), 1).to(DEV), bf16((L, 3, Hkv, n, d), 2).to(DEV)
    idx = torch.arange(10, dtype=torch.int32, device=DEV).expand(L, 3, Hkv, 10).contiguous()

    def go(c, seqs, write, idx=idx, pos=(0,) * 6):
        b = len(seqs)
        for s, slot in write:
            for h in range(Hkv):
                for j in range(10):
                    t = int(idx[0, s, h, j])
                    c.write(slot, 0, h, j, f64(k[0, s, h, min(t, n - 1)]), f64(v[0, s, h, min(t, n - 1)]), empty=t >= n)
        st = new_status()
        R.kv_compact_q4(R.Batch(L, b, Hkv, Hkv, d, n), k[:, :b], v[:, :b], idx[:, :b].contiguous(), 0.25, c.pool, c.pages,
                        i32(list(pos)), seqs=i32(seqs), status=st)
        c.check_pool()
        return st.item()

    assert go(fresh(), [5, 2], [(0, 5), (1, 2)]) == 0
    assert go(fresh(), [5, 2, 5], [(0, 5), (1, 2)]) == R.STATUS_BAD_INDEX
    assert go(fresh(), [6, 2, -1], [(1, 2)]) == R.STATUS_BAD_INDEX
    assert go(fresh(), [5, 2], [(0, 5)], pos=(0, 0, -1, 0, 0, 0)) == 0
    assert go(fresh(), [5, 1], [(0, 5)]) == R.STATUS_BAD_INDEX                    # slot 1 has no page
    assert go(fresh(), [5, 2], [(0, 5)], pos=(0, 0, 4 * P, 0, 0, 0)) == R.STATUS_BAD_INDEX   # past the table
    assert go(fresh(), [5, 2], [(0, 5)], pos=(0, 0, 2 ** 31 - 1, 0, 0, 0)) == R.STATUS_BAD_INDEX
    far = idx.clone()
    far[0, 0, 1, 4] = n
    assert go(fresh(), [5, 2], [(0, 5), (1, 2)], idx=far) == R.STATUS_BAD_INDEX


# ------------------------------------------------------------------ rows read ----

@pytest.mark.parametrize("d, P, lens, start, rows", [
    (128, 16, [0, 1, 16, 17, 50], None, 50), (64, 32, [100, 31, 32], [0, 31, 5], 33), (128, 64, [130, 70], [129, 0], 1),
    (64, 16, [40, 40], [39, 40], 7)])
def test_expand(d, P, lens, start, rows):
    L, Hkv, b = 2, 2, len(lens)
    c = Cache(b, pages_for(lens, P), P, -(-max(lens) // P) + 2, L, Hkv, d).fill(lens, shuffle=4).random_rows(3, empty=0.2)
    # outputs whose heads lie inside the token rows
    out = [torch.full((L, b, rows, Hkv, d), 7.0, dtype=torch.bfloat16, device=DEV).transpose(2, 3) for _ in "kv"]
    st = new_status()
    R.kv_expand_q4(c.pool, c.pages, *out, start=None if start is None else i32(start), status=st)
    for s in range(b):
        a = 0 if start is None else start[s]
        for l in range(L):
            for h in range(Hkv):
                for o, want in zip(out, c.rows(s, l, h)):
                    m = max(0, min(rows, lens[s] - a))
                    assert torch.equal(o[l, s, h, :m].cpu(), torch.from_numpy(want[a:a + m]).float().bfloat16())
                    assert (o[l, s, h, m:] == 7.0).all()
    assert st.item() == 0


# ------------------------------------------------------------------ attention ----

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
def test_attention_over_short_and_ragged_lengths(d, G):
    lens = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 130]
    L, Hkv, P = 2, 2, (16, 48, 64)[G % 3]
    c = Cache(len(lens), pages_for(lens, P), P, -(-max(lens) // P) + 1, L, Hkv, d).fill(lens, shuffle=G).random_rows(G)
    q = bf16((L, len(lens), Hkv * G, d), 9)
    out = torch.full((L, len(lens), Hkv * G, d), 7.0, device=DEV)
    st = new_status()
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out, status=st)
    check_attention(out, q, c)
    assert st.item() == 0


@pytest.mark.parametrize("lens, Hkv, L", [([2000], 1, 1), ([5000, 3, 700], 2, 1), ([900] * 3, 8, 2), ([16] * 40, 4, 2),
                                          ([0, 1200, 0, 0, 33, 0], 1, 2), ([0, 300] + [0] * 9 + [290] * 5, 8, 3)])
def test_attention_rows_shared_among_ctas(lens, Hkv, L):
    d, G, P = 128, 4, 64
    c = Cache(len(lens), pages_for(lens, P), P, -(-max(lens) // P), L, Hkv, d).fill(lens, shuffle=1).random_rows(5)
    q = bf16((L, len(lens), Hkv * G, d), 9, 3.0)
    out = torch.empty((L, len(lens), Hkv * G, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)
    again = torch.empty_like(out)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, again)
    assert torch.equal(out, again)                            # (the same bits every time)


@pytest.mark.parametrize("d, G", [(64, 4), (128, 7)])
def test_attention_skips_empty_slots(d, G):
    """Empty slots anywhere; one sequence of nothing else gives zeros."""
    lens = [70, 40, 5]
    c = Cache(3, pages_for(lens, 16), 16, 6, 1, 2, d).fill(lens, shuffle=1).random_rows(8, empty=0.5)
    for r in range(40):
        for h in range(2):
            c.write(1, 0, h, r, np.zeros(d), np.zeros(d), empty=True)
    c.pool.copy_(torch.from_numpy(c.want))
    q = bf16((1, 3, 2 * G, d), 2)
    out = torch.full((1, 3, 2 * G, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)
    assert (out[:, 1] == 0).all()


@pytest.mark.parametrize("qs, ks, vs", [(1.0, 1.0, 2.0 ** 60), (1.0, 1.0, 2.0 ** -60), (2.0 ** 40, 2.0 ** -40, 1.0),
                                        (2.0 ** -40, 2.0 ** 40, 1.0), (8.0, 4.0, 1.0)])
def test_attention_over_magnitudes(qs, ks, vs):
    """Queries, keys and values far from one; logits that reach hundreds."""
    d, G, Hkv = 128, 3, 2
    lens = [150, 20]
    c = Cache(2, pages_for(lens, 32), 32, 6, 1, Hkv, d).fill(lens)
    for s, n in enumerate(lens):
        for h in range(Hkv):
            k, v = f64(bf16((n, d), 5 + s, ks)), f64(bf16((n, d), 8 + h, vs))
            for r in range(n):
                # values that differ by 2^20 from row to row
                c.write(s, 0, h, r, k[r], v[r] * 2.0 ** (-20 * (r % 2)))
    c.pool.copy_(torch.from_numpy(c.want))
    q = bf16((1, 2, Hkv * G, d), 9, qs)
    q[0, 0, 0, 1::2] = 0
    out = torch.empty((1, 2, Hkv * G, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


def test_attention_keeps_a_heavy_tail():
    """One key takes half of the weight, thousands share the rest: their small
    probabilities must not be rounded away."""
    d, n = 64, 6000
    c = Cache(1, pages_for([n], 64), 64, 94, 1, 1, d).fill([n])
    q = torch.zeros(1, 1, 1, d)
    q[..., 0] = 8.0
    q = q.bfloat16()
    k = np.zeros((n, d))
    k[100, 0] = float(torch.tensor(np.log(n) * d ** 0.5 / 8.0).bfloat16())
    v = f64(bf16((n, d), 4))
    for r in range(n):
        c.write(0, 0, 0, r, k[r], v[r])
    c.pool.copy_(torch.from_numpy(c.want))
    out = torch.empty((1, 1, 1, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


def test_attention_nonfinite_rows():
    """A NaN among the kept rows shows in the outputs that depend on it, and
    only there; rows past the end never do (they hold NaN scales here)."""
    d, G = 128, 2
    lens = [40, 21, 21]
    c = Cache(3, 12, 16, 3, 1, 1, d).fill(lens)
    c.want[...] = 0xFF                                        # every scale a NaN
    for s, n in enumerate(lens):
        for r in range(n):
            k, v = f64(bf16(d, r)), f64(bf16(d, 50 + r))
            if s == 1 and r == 7:
                v[70] = np.inf
            if s == 2 and r == 7:
                k[3] = np.nan
            c.write(s, 0, 0, r, k, v)
    c.pool.copy_(torch.from_numpy(c.want))
    q = bf16((1, 3, G, d), 1)
    out = torch.empty((1, 3, G, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    got = out.cpu()
    assert torch.isfinite(got[0, 0]).all()
    assert torch.isnan(got[0, 1, :, 64:96]).all() and torch.isfinite(got[0, 1, :, :64]).all() \
        and torch.isfinite(got[0, 1, :, 96:]).all()
    assert torch.isnan(got[0, 2]).all()
    check_attention(out[:, :1], q[:, :1], c)


def test_attention_of_a_batch_of_slots():
    """Sequences in any order, one twice, one out of range (zeros); a table
    entry without a page: its rows are absent; strided queries; a scale."""
    d, G, Hkv, P = 64, 4, 2, 16
    lens = [50, 0, 33, 20]
    c = Cache(4, 20, P, 5, 2, Hkv, d).fill(lens, shuffle=6).random_rows(1)
    seqs = [3, 0, 3, 9, 2, 1, -1]
    q = bf16((len(seqs), 2, 2 * Hkv * G, d), 3).transpose(0, 1)[:, :, ::2]
    out = torch.full((2, len(seqs), Hkv * G, d), 7.0, device=DEV)
    st = new_status()
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out, scale=0.3, seqs=i32(seqs), status=st)
    check_attention(out, q, c, seqs=seqs, scale=0.3)
    assert st.item() == R.STATUS_BAD_INDEX
    # slot 0 without its second page
    c.pages.table[0, 1] = -1
    st.zero_()
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out, scale=0.3, seqs=i32(seqs), status=st)
    assert st.item() == R.STATUS_BAD_INDEX
    for l in range(2):
        for h in range(Hkv):
            k, v, e = c.rows(0, l, h)
            e[P:2 * P] = True
            want = Q.attention(f64(q[l, 1, h * G:(h + 1) * G]), k, v, e, 0.3)[0]
            assert np.abs(f64(out[l, 1, h * G:(h + 1) * G]) - want).max() < 1e-5
    c.pages.lens[2] = 5 * P + 1                               # longer than the table
    st.zero_()
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out, seqs=i32(seqs), status=st)
    assert st.item() == R.STATUS_BAD_INDEX
    torch.cuda.synchronize()


# ----------------------------------------------------------------------- book ----

@pytest.mark.parametrize("seed", range(6))
def test_book_follows_the_oracle(seed):
    """Random reserves, forks, frees and packs; every copied page's rows."""
    rng = np.random.default_rng(seed)
    n_seqs, n_pages, P, M = int(rng.integers(1, 9)), int(rng.integers(6, 60)), int(rng.choice([16, 32])), 9
    c = Cache(n_seqs, n_pages, P, M, 2, 2, 64, seed=seed)
    ws = R.pages_workspace(c.pages)
    pos = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
    for step in range(25):
        st = new_status()
        op = rng.choice(["reserve", "reserve", "reserve", "fork", "pack"])
        if op == "reserve":
            add = [int(x) for x in rng.choice([0, 1, 1, 5, P, 3 * P, -1], n_seqs)]
            want, copies = c.book.reserve(add)
            R.kv_pages_reserve(c.pages, c.pool, i32(add), pos, ws=ws, status=st)
            assert pos.tolist() == want
            for a, z, rows in copies:
                recs = -(-rows // 16)
                c.want[:, z, :, :recs] = c.want[:, a, :, :recs]
            short = any(w < 0 <= x for w, x in zip(want, add))
            assert st.item() == (R.STATUS_NO_PAGES if short else 0) + (R.STATUS_BAD_INDEX if min(add) < 0 else 0)
        elif op == "fork":
            parent = [int(x) for x in rng.choice([-1] + list(range(n_seqs)) * 2, n_seqs)]
            if step % 7 == 0:
                parent[0] = n_seqs
            c.book.fork(parent)
            R.kv_pages_fork(c.pages, i32(parent), ws=ws, status=st)
            assert st.item() == (R.STATUS_BAD_INDEX if step % 7 == 0 else 0)
        else:
            n, moves = c.book.pack()
            live = i32([0])
            R.kv_pages_pack(c.pages, c.pool, n_live=live, ws=ws, status=st)
            assert live.item() == n and st.item() == 0
            for a, z in moves:
                c.want[:, z] = c.want[:, a]
        c.check_book()
        c.check_pool()


def test_book_of_many_pages():
    """More pages than one round of the scan looks at, more slots than threads."""
    n_seqs, n_pages, P = 1500, 30011, 16
    rng = np.random.default_rng(4)
    c = Cache(n_seqs, n_pages, P, 40, 1, 1, 64)
    ws = R.pages_workspace(c.pages)
    pos = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
    for step in range(3):
        add = [int(x) for x in rng.integers(0, 14 * P, n_seqs)]
        want, copies = c.book.reserve(add)
        R.kv_pages_reserve(c.pages, c.pool, i32(add), pos, ws=ws)
        assert pos.tolist() == want
        c.check_book()
        parent = np.arange(n_seqs)
        drop = rng.random(n_seqs) < 0.4
        parent[drop] = rng.integers(-1, n_seqs, int(drop.sum()))
        c.book.fork(parent.tolist())
        R.kv_pages_fork(c.pages, i32(parent.tolist()), ws=ws)
        c.check_book()
        n, _ = c.book.pack()
        live = i32([0])
        R.kv_pages_pack(c.pages, c.pool, n_live=live, ws=ws)
        assert live.item() == n
        c.check_book()


# ------------------------------------------------------------------- together ----

@pytest.mark.parametrize("d, G", [(128, 4), (64, 8)])
def test_prompt_to_samples(d, G):
    """A prompt scored, selected and compacted into pages, forked into samples,
    tokens appended (the shared last page copied), attention after each, two
    samples freed, the pool packed, a second round of scoring on what is left:
    the cache's bytes and the outputs follow the oracle all the way."""
    L, Hkv, n, P, B, W = 2, 2, 600, 32, 0.2, 16
    w = I.Workload("q4", "snapkv", L, 1, Hkv * G, Hkv, d, n, W, 7, (B,), 4, (3, 5), (1, 3))
    roles = I.workload_roles(w, 3)
    k, v = I.make_kv(w, roles, 3, device=DEV)
    qw = I.make_q_window(w, 3, device=DEV)
    batch = R.Batch(L, 1, Hkv * G, Hkv, d, n)
    scores = torch.empty(batch.score_shape(), device=DEV)
    R.snapkv_score(batch, qw, k, W, 7, scores)
    idx = torch.empty(batch.kept_shape(B), dtype=torch.int32, device=DEV)
    R.role_alloc_select(batch, scores, torch.as_tensor(roles, device=DEV),
                        R.select_params(B, I.PAPER_ALPHA, alpha_key=0.02, key_role=I.ROLE_KEY), idx)
    m = idx.shape[-1]
    c = Cache(4, 40, P, 8, L, Hkv, d, seed=3)
    pos = torch.zeros(4, dtype=torch.int32, device=DEV)
    st = new_status()

    def reserve(add):
        want, copies = c.book.reserve(add)
        R.kv_pages_reserve(c.pages, c.pool, i32(add), pos, status=st)
        for a, z, rows in copies:
            c.want[:, z, :, :-(-rows // 16)] = c.want[:, a, :, :-(-rows // 16)]
        return want

    reserve([0, m, 0, 0])
    R.kv_compact_q4(batch, k, v, idx, B, c.pool, c.pages, pos, seqs=i32([1]), status=st)
    kept = idx.cpu().numpy()
    for l in range(L):
        for h in range(Hkv):
            for j, t in enumerate(kept[l, 0, h]):
                c.write(1, l, h, j, f64(k[l, 0, h, t]), f64(v[l, 0, h, t]))
    c.check_pool()
    parent = [1, 1, 1, -1]
    c.book.fork(parent)
    R.kv_pages_fork(c.pages, i32(parent), status=st)
    for step in range(3):
        kn, vn = bf16((L, 4, Hkv, 1, d), 20 + step), bf16((L, 4, Hkv, 1, d), 30 + step)
        want = reserve([1, 1, 1, 0])
        R.kv_append_q4(c.pool, c.pages, kn.to(DEV), vn.to(DEV), pos, count=i32([1, 1, 1, 0]), status=st)
        for s in range(3):
            for l in range(L):
                for h in range(Hkv):
                    c.write(s, l, h, want[s], f64(kn[l, s, h, 0]), f64(vn[l, s, h, 0]))
        c.check_book()
        c.check_pool()
        q = bf16((L, 4, Hkv * G, d), 40 + step)
        out = torch.empty((L, 4, Hkv * G, d), device=DEV)
        R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out, status=st)
        check_attention(out, q, c)
    parent = [-1, 1, -1, 3]
    c.book.fork(parent)
    R.kv_pages_fork(c.pages, i32(parent), status=st)
    live = i32([0])
    R.kv_pages_pack(c.pages, c.pool, n_live=live, status=st)
    count, moves = c.book.pack()
    for a, z in moves:
        c.want[:, z] = c.want[:, a]
    assert live.item() == count == -(-(m + 3) // P)
    c.check_book()
    c.check_pool()
    assert st.item() == 0
    # what is left, scored again
    ko, vo = (torch.zeros((L, 1, Hkv, m + 3, d), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    R.kv_expand_q4(c.pool, c.pages, ko, vo, seqs=i32([1]))
    for l in range(L):
        for h in range(Hkv):
            assert torch.equal(ko[l, 0, h].cpu(), torch.from_numpy(c.rows(1, l, h)[0]).float().bfloat16())
    again = R.Batch(L, 1, Hkv * G, Hkv, d, m + 3)
    s2 = torch.empty(again.score_shape(), device=DEV)
    R.snapkv_score(again, qw, ko, W, 1, s2)
    assert abs(s2[0, 0, 0].double().sum().item() - W * G) < 1e-3 * W * G


def step_calls(c, q, kn, vn, add, pos, out, ws, dws, st):
    R.kv_pages_reserve(c.pages, c.pool, add, pos, ws=ws, status=st)
    R.kv_append_q4(c.pool, c.pages, kn, vn, pos, status=st)
    R.decode_attention_q4(q, c.pool, c.pages, out, ws=dws, status=st)


def test_steps_captured_in_a_graph():
    """Decode steps replayed from one graph (lengths and pages move on the
    device) leave what the same calls made one by one leave; two graphs share
    the workspaces."""
    L, b, Hkv, G, d, P = 1, 3, 2, 4, 128, 16
    lens = [14, 40, 0]
    def fresh():
        return Cache(b, 20, P, 6, L, Hkv, d).fill(lens, shuffle=2).random_rows(3)
    q, kn, vn = (bf16((L, b, Hkv * G, d), 1).to(DEV), bf16((L, b, Hkv, 1, d), 2).to(DEV),
                 bf16((L, b, Hkv, 1, d), 3).to(DEV))
    add, st = i32([1] * b), new_status()
    eager, graphed = fresh(), fresh()
    ws, dws = R.pages_workspace(eager.pages), R.decode_q4_workspace(L, b, Hkv * G, Hkv, d)
    pos = torch.zeros(b, dtype=torch.int32, device=DEV)
    outs = []
    for _ in range(6):
        out = torch.empty((L, b, Hkv * G, d), device=DEV)
        step_calls(eager, q, kn, vn, add, pos, out, ws, dws, st)
        outs.append(out)
    gout = [torch.empty((L, b, Hkv * G, d), device=DEV) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    for g, o in zip(graphs, gout):
        with torch.cuda.graph(g):
            step_calls(graphed, q, kn, vn, add, pos, o, ws, dws, st)
    for i in range(6):
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(gout[i % 2], outs[i])
    assert torch.equal(graphed.pages.state, eager.pages.state) and torch.equal(graphed.pool, eager.pool)
    assert st.item() == 0


def test_book_calls_captured_in_a_graph():
    """Fork, pack and expansion replayed: a cycle of parents that comes back to
    where it began after three replays."""
    d, P, lens = 64, 16, [40, 7, 100]
    c = Cache(3, 14, P, 8, 1, 2, d).fill(lens, shuffle=5).random_rows(2)
    ws = R.pages_workspace(c.pages)
    parent, live, st = i32([1, 2, 0]), i32([0]), new_status()
    out = [torch.zeros((1, 3, 2, 100, d), dtype=torch.bfloat16, device=DEV) for _ in "kv"]

    def calls():
        R.kv_pages_fork(c.pages, parent, ws=ws, status=st)
        R.kv_pages_pack(c.pages, c.pool, n_live=live, ws=ws, status=st)
        R.kv_expand_q4(c.pool, c.pages, *out, status=st)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        calls()
    rows = [[c.rows(s, 0, h) for h in range(2)] for s in range(3)]
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert live.item() == sum(-(-n // P) for n in lens) and st.item() == 0
        for s in range(3):
            of = (s + i + 1) % 3
            for h in range(2):
                for o, want in zip(out, rows[of][h]):
                    assert torch.equal(o[0, s, h, :lens[of]].cpu(), torch.from_numpy(want).float().bfloat16())
    assert c.pages.lens.tolist() == lens


def test_more_sequences_than_threads():
    """600 sequences, most of them short or empty, behind tables long enough
    that rows are shared among CTAs."""
    rng = np.random.default_rng(0)
    b, P, d, Hkv, G = 600, 16, 64, 1, 2
    lens = [int(x) for x in rng.choice([0, 1, 15, 16, 40], b)]
    lens[500] = 700
    c = Cache(b, pages_for(lens, P), P, 60, 1, Hkv, d).fill(lens, shuffle=3).random_rows(1)
    q = bf16((1, b, Hkv * G, d), 9)
    out = torch.full((1, b, Hkv * G, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


def test_offsets_past_32_bits():
    """Layers 3 GB apart, the last page of each near its end."""
    d, P, Hkv, n, far = 64, 16, 2, 21, 3 << 30
    page = R.q4_pool_shape(2, 1, Hkv, d, P)[2:]
    size = page[0] * page[1] * page[2]
    n_pages = far // size
    pages = R.Pages(1, n_pages, P, 2)
    buf = torch.empty(2 * far, dtype=torch.uint8, device=DEV)
    pool = buf.as_strided((2, n_pages) + page, (far, size, page[1] * page[2], page[2], 1))
    pages.table.copy_(i32([[n_pages - 1, n_pages - 3]]))
    pages.refs[n_pages - 1] = pages.refs[n_pages - 3] = 1
    pages.lens.fill_(n)
    k, v = bf16((2, 1, Hkv, n, d), 1), bf16((2, 1, Hkv, n, d), 2)
    st = new_status()
    R.kv_append_q4(pool, pages, k.to(DEV), v.to(DEV), i32([0]), status=st)
    out = [torch.zeros((2, 1, Hkv, n, d), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    R.kv_expand_q4(pool, pages, *out, status=st)
    kv = [Q.values(f64(x)) for x in (k, v)]
    for o, want in zip(out, kv):
        assert torch.equal(o.cpu(), torch.from_numpy(want).float().bfloat16())
    q = bf16((2, 1, Hkv, d), 3)
    got = R.decode_attention_q4(q.to(DEV), pool, pages, torch.empty((2, 1, Hkv, d), device=DEV), status=st)
    for l in range(2):
        for h in range(Hkv):
            want = Q.attention(f64(q[l, 0, h:h + 1]), kv[0][l, 0, h], kv[1][l, 0, h], np.zeros(n, bool), d ** -0.5)[0]
            assert np.abs(f64(got[l, 0, h:h + 1]) - want).max() < 1e-5
    live = i32([0])
    pages.refs[5] = 1                                          # (somebody else's page: moves to 0, the lowest)
    R.kv_pages_pack(pages, pool, n_live=live, status=st)
    assert live.item() == 3 and pages.table.tolist() == [[2, 1]] and st.item() == 0
    for o in out:
        o.zero_()
    R.kv_expand_q4(pool, pages, *out)
    for o, want in zip(out, kv):
        assert torch.equal(o.cpu(), torch.from_numpy(want).float().bfloat16())


def test_calls_behind_a_call_on_another_stream():
    """A step's calls on a stream of their own, with workspaces of their own,
    behind work that writes their inputs late on the same stream."""
    L, b, Hkv, G, d, P = 1, 2, 2, 4, 128, 16
    c = Cache(b, 12, P, 4, L, Hkv, d).fill([20, 31], shuffle=2).random_rows(3)
    q, kn, vn = (bf16((L, b, Hkv * G, d), 1).to(DEV), bf16((L, b, Hkv, 1, d), 2), bf16((L, b, Hkv, 1, d), 3))
    late = [torch.zeros_like(x, device=DEV) for x in (kn, vn)]
    src = [x.to(DEV) for x in (kn, vn)]
    add = i32([1, 1])
    pos = torch.zeros(b, dtype=torch.int32, device=DEV)
    out = torch.empty((L, b, Hkv * G, d), device=DEV)
    big = torch.empty(1 << 28, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(4):
            big.zero_()
        for x, y in zip(late, src):
            x.copy_(y)
    want, _ = c.book.reserve([1, 1])
    R.kv_pages_reserve(c.pages, c.pool, add, pos, stream=s)
    R.kv_append_q4(c.pool, c.pages, *late, pos, stream=s)
    R.decode_attention_q4(q, c.pool, c.pages, out, stream=s)
    torch.cuda.synchronize()
    for x in range(b):
        for h in range(Hkv):
            c.write(x, 0, h, want[x], f64(kn[0, x, h, 0]), f64(vn[0, x, h, 0]))
    c.check_book()
    c.check_pool()
    check_attention(out, q.cpu(), c)


def test_tensors_elsewhere_are_refused():
    d, P = 64, 16
    c = Cache(1, 3, P, 2, 1, 1, d).fill([5]).random_rows(1)
    q, out = bf16((1, 1, 1, d), 1), torch.empty((1, 1, 1, d), device=DEV)
    with pytest.raises(ValueError, match="current device"):
        R.decode_attention_q4(q, c.pool, c.pages, out)
    with pytest.raises(ValueError, match="current device"):
        R.kv_pages_fork(c.pages, torch.zeros(1, dtype=torch.int32))
    batch = R.Batch(1, 1, 1, 1, d, 8)
    k = bf16((1, 1, 1, 8, d), 1).to(DEV)
    idx = torch.zeros((1, 1, 1, 4), dtype=torch.int32, device=DEV)
    for kk, ii in ((k[..., :7, :], idx), (k, idx[..., :3]), (k, idx.long())):
        with pytest.raises(ValueError):
            R.kv_compact_q4(batch, kk, k, ii, 0.5, c.pool, c.pages, i32([0]))


def test_reads_on_two_streams():
    """Attention and expansion of one cache at the same time, each on a stream
    of its own and with a workspace of its own."""
    L, b, Hkv, G, d, P = 1, 4, 4, 4, 128, 32
    lens = [400, 33, 700, 1]
    c = Cache(b, pages_for(lens, P), P, 22, L, Hkv, d).fill(lens, shuffle=2).random_rows(3)
    q = bf16((L, b, Hkv * G, d), 1).to(DEV)
    want = R.decode_attention_q4(q, c.pool, c.pages, torch.empty((L, b, Hkv * G, d), device=DEV))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        out = torch.empty((L, b, Hkv * G, d), device=DEV)
        streams[i % 2].wait_stream(torch.cuda.current_stream())
        got.append(R.decode_attention_q4(q, c.pool, c.pages, out, stream=streams[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_pools_of_other_strides():
    """A pool held page by page ([n_pages][L]), and one layer of it."""
    L, b, Hkv, G, d, P = 3, 2, 2, 2, 64, 16
    lens = [30, 17]
    c = Cache(b, 8, P, 3, L, Hkv, d).fill(lens, shuffle=2).random_rows(3)
    q = bf16((L, b, Hkv * G, d), 1).to(DEV)
    want = R.decode_attention_q4(q, c.pool, c.pages, torch.empty((L, b, Hkv * G, d), device=DEV))
    check_attention(want, q, c)
    by_page = c.pool.transpose(0, 1).contiguous().transpose(0, 1)
    got = R.decode_attention_q4(q, by_page, c.pages, torch.empty_like(want))
    assert torch.equal(got, want)
    for l in range(L):
        one = R.decode_attention_q4(q[l:l + 1], by_page[l:l + 1], c.pages, torch.empty_like(want[:1]))
        assert torch.allclose(one, want[l:l + 1], rtol=1e-5, atol=1e-6)


def test_batch_lengths_elsewhere_are_refused():
    """A packed batch whose device copy of its offsets is on the host."""
    d, P = 64, 16
    c = Cache(1, 3, P, 2, 1, 1, d).fill([5]).random_rows(1)
    batch = R.Batch(1, 1, 1, 1, d, 8, seqlens=[8], device="cpu")
    k = bf16((1, 8, 1, d), 1).to(DEV)
    idx = torch.zeros(4, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="current device"):
        R.kv_compact_q4(batch, k, k, idx, 0.5, c.pool, c.pages, i32([0]))


def test_more_rows_asked_for_than_any_sequence_has():
    """2^31 - 1 rows to read back or to append, of which the lengths and counts
    leave a few."""
    d, P, n, top = 64, 16, 21, (1 << 31) - 1
    c = Cache(1, 3, P, 3, 1, 1, d).fill([n], shuffle=1).random_rows(1)
    lib, st = R.lib(), new_status()
    out = torch.zeros((2, n, d), dtype=torch.bfloat16, device=DEV)
    t = [R.Tensor(x.data_ptr(), 0, 0, 0, d) for x in out]
    pd, pg = R.pool_desc(c.pool, c.pages), c.pages.desc
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.kv_expand_q4(ctypes.byref(pd), ctypes.byref(pg), None, 1, None, top, *t, st.data_ptr(), stream) == 0
    k, v, _ = c.rows(0, 0, 0)
    for got, want in zip(out.cpu(), (k, v)):
        assert torch.equal(got, torch.from_numpy(want).float().bfloat16())
    new = bf16((2, 3, d), 5)
    x = new.to(DEV)
    t = [R.Tensor(y.data_ptr(), 0, 0, 0, d) for y in x]
    count, pos = i32([3]), i32([7])
    assert lib.kv_append_q4(ctypes.byref(pd), ctypes.byref(pg), None, 1, *t, top, count.data_ptr(), pos.data_ptr(),
                            st.data_ptr(), stream) == 0
    for i in range(3):
        c.write(0, 0, 0, 7 + i, f64(new[0, i]), f64(new[1, i]))
    c.check_pool()
    assert st.item() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [5, 6, 7])
def test_append_around_the_choice_of_kernel(d, T):
    """A row to some lanes, or records to a warp: the same bytes."""
    L, Hkv, b, P = 2, 2, 5, 16
    pos = [0, 3, 8, 13, 16]
    lens = [p + T for p in pos]
    c = Cache(b, pages_for(lens, P), P, 3, L, Hkv, d, seed=T).fill(lens, shuffle=1)
    k, v = bf16((L, b, Hkv, T, d), 1), bf16((L, b, Hkv, T, d), 2, 3.0)
    for s in range(b):
        for i in range(T):
            for l in range(L):
                for h in range(Hkv):
                    c.write(s, l, h, pos[s] + i, f64(k[l, s, h, i]), f64(v[l, s, h, i]))
    R.kv_append_q4(c.pool, c.pages, k.to(DEV), v.to(DEV), i32(pos))
    c.check_pool()


@pytest.mark.parametrize("pages", [12, 13])
def test_attention_around_the_choice_of_sharing(pages):
    """Units of as many rows as go to a CTA each, and of more."""
    L, Hkv, G, d, P = 1, 2, 3, 128, 32
    lens = [pages * P, pages * P - 1, 0, 1, 5 * P + 3]
    c = Cache(5, pages_for(lens, P), P, pages, L, Hkv, d).fill(lens, shuffle=2).random_rows(4)
    q = bf16((L, 5, Hkv * G, d), 9)
    out = torch.full((L, 5, Hkv * G, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


@pytest.mark.parametrize("units", [114, 115])
def test_attention_around_the_choice_of_join(units):
    """Cut units joined one by one, or by the CTA that begins them."""
    d, P, n = 64, 64, 900
    c = Cache(units, units * 15, P, 15, 1, 1, d).fill([n if s % 7 else 0 for s in range(units)], shuffle=2)
    k, v = (bf16((1, units, 1, n, d), x).to(DEV) for x in (1, 2))
    R.kv_append_q4(c.pool, c.pages, k, v, i32([0 if s % 7 else -1 for s in range(units)]))
    c.want = c.pool.cpu().numpy()
    q = bf16((1, units, 2, d), 9)
    out = torch.full((1, units, 2, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


@pytest.mark.parametrize("max_pages", [1024, 1025])
def test_fork_around_the_choice_of_launches(max_pages):
    """Tables that a cluster forks in one launch, and larger ones."""
    n_seqs, P = 24, 16
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, max_pages * P + 1, n_seqs)]
    lens[3], lens[4] = max_pages * P, 0
    c = Cache(n_seqs, pages_for(lens, P), P, max_pages, 1, 1, 64).fill(lens, shuffle=1)
    parent = [int(x) for x in rng.integers(-1, n_seqs, n_seqs)]
    parent[4], parent[5], parent[6] = 3, 5, -1
    c.book.fork(parent)
    R.kv_pages_fork(c.pages, i32(parent))
    c.check_book()


def test_the_largest_batch():
    """4096 sequences, and as many without a row."""
    rng = np.random.default_rng(0)
    b, P, d, G = 4096, 16, 64, 2
    lens = [int(x) for x in rng.choice([0, 1, 16, 17], b, p=[0.4, 0.3, 0.2, 0.1])]
    lens[4000] = 600
    c = Cache(b, pages_for(lens, P), P, 40, 1, 1, d).fill(lens, shuffle=3).random_rows(1)
    q = bf16((1, b, G, d), 9)
    out = torch.full((1, b, G, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)
    c.pages.lens.zero_()
    out.fill_(7.0)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    assert not out.any()


def test_decode_from_two_threads():
    """Calls over batches of very different sizes, each from a thread and on a
    stream of its own."""
    import threading
    d, P, G = 64, 16, 4
    sizes = [3, 1500]
    caches = [Cache(b, 2 * b, P, 40, 1, 1, d).fill([30] * b, shuffle=1).random_rows(1) for b in sizes]
    qs = [bf16((1, b, G, d), 9).to(DEV) for b in sizes]
    want = [R.decode_attention_q4(q, c.pool, c.pages, torch.empty(q.shape, device=DEV)) for q, c in zip(qs, caches)]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    got, errors = [None] * 2, []

    def work(i):
        try:
            with torch.cuda.stream(streams[i]):
                outs = [torch.empty(qs[i].shape, device=DEV) for _ in range(200)]
                for o in outs:
                    R.decode_attention_q4(qs[i], caches[i].pool, caches[i].pages, o)
            got[i] = outs
        except Exception as e:                        # (a thread's own would be lost)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert all(torch.equal(o, w) for outs, w in zip(got, want) for o in outs)


@pytest.mark.parametrize("L, b, Hkv, d", [(8, 256, 15, 64), (20, 256, 6, 128)])
def test_single_rows_of_large_batches(L, b, Hkv, d):
    """So many that a warp takes several heads: appended to chosen slots at every
    place in a record, and compacted from prompts that keep two rows, one of them
    an empty slot, in other slots."""
    P = 16
    rng = np.random.default_rng(3)
    pos = [int(x) for x in rng.integers(0, 14, b)]
    c = Cache(b, b + 3, P, 1, L, Hkv, d, seed=1).fill([p + 2 for p in pos], shuffle=1)
    slots = [int(x) for x in rng.permutation(b)]
    pos[slots[5]] = -1
    k, v = bf16((L, b, Hkv, 1, d), 1), bf16((L, b, Hkv, 1, d), 2, 3.0)
    k64, v64 = f64(k), f64(v)
    R.kv_append_q4(c.pool, c.pages, k.to(DEV), v.to(DEV), i32(pos), seqs=i32(slots))
    for s in range(b):
        for l in range(L):
            for h in range(Hkv):
                if pos[slots[s]] >= 0:
                    c.write(slots[s], l, h, pos[slots[s]], k64[l, s, h, 0], v64[l, s, h, 0])
    c.check_pool()
    n = 8
    batch = R.Batch(L, b, Hkv, Hkv, d, n)
    k, v = bf16((L, b, Hkv, n, d), 5), bf16((L, b, Hkv, n, d), 6)
    k64, v64 = f64(k), f64(v)
    idx = torch.from_numpy(rng.integers(0, n, (L, b, Hkv, 2))).int()
    idx[:, ::3, :, 1] = -1
    st = new_status()
    R.kv_compact_q4(batch, k.to(DEV), v.to(DEV), idx.to(DEV), 0.25, c.pool, c.pages, i32(pos), status=st)
    for s in range(b):
        for l in range(L):
            for h in range(Hkv):
                for j in range(2 if pos[s] >= 0 else 0):
                    i = int(idx[l, s, h, j])
                    c.write(s, l, h, pos[s] + j, k64[l, s, h, max(i, 0)], v64[l, s, h, max(i, 0)], i < 0)
    c.check_pool()
    assert st.item() == 0


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("seqs", [1, 120])
@pytest.mark.parametrize("where", ["keys", "values"])
def test_a_part_of_no_weight_keeps_its_nan(seqs, where):
    """Rows of a sequence shared by several CTAs: NaN keys that fill a CTA's part,
    and a NaN value in a part whose logits lie hundreds below the others', show in
    the outputs as they do where one CTA has all rows.  Units begin with 32 to
    256 such rows, so that some of them fill a part and no more."""
    d, P, G, n = 64, 64, 2, 2048 if seqs == 1 else 900
    Hkv = 8 if seqs == 1 else 1
    units = seqs * Hkv
    assert (4 * units <= 3 * sms()) == (seqs == 1)            # joined by unit, or by the CTA that begins one
    lens = [n] * seqs
    c = Cache(seqs, pages_for(lens, P), P, -(-n // P), 1, Hkv, d).fill(lens, shuffle=2)
    k, v = torch.full((1, seqs, Hkv, n, d), 8.0), bf16((1, seqs, Hkv, n, d), 2).float()
    first = torch.tensor([32 * (1 + (u // 8 if seqs > 1 else u) % 8) for u in range(units)]).view(seqs, Hkv)
    for s in range(seqs):
        for h in range(Hkv):
            if where == "keys":
                k[0, s, h, :first[s, h]] = float("nan")
            else:
                k[0, s, h, :first[s, h]] = 0.0
                v[0, s, h, 5, 3] = float("nan")
    R.kv_append_q4(c.pool, c.pages, k.bfloat16().to(DEV), v.bfloat16().to(DEV), i32([0] * seqs))
    q = torch.full((1, seqs, Hkv * G, d), 8.0).bfloat16()
    out = torch.empty(q.shape, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    got = out.cpu()
    if where == "keys":
        assert torch.isnan(got).all(), f"{int(torch.isfinite(got).any(-1).sum())} heads are finite"
    else:
        assert torch.isnan(got[..., :32]).all(), "a NaN value does not show"
        assert torch.isfinite(got[..., 32:]).all()


@pytest.mark.parametrize("n", [384, 4000])
@pytest.mark.parametrize("before, after", [(0.0, 2.0 ** 45), (2.0 ** -60, 2.0 ** 60), (2.0 ** 45, 0.0),
                                           (2.0 ** 99, 2.0 ** -99), (2.0 ** -99, 2.0 ** 99), (0.0, 2.0 ** 124)])
def test_attention_over_values_that_change_in_size(n, before, after):
    """Rows of values of one size, then as many of another: all count with the
    weights that their keys give them, in one CTA and over several."""
    d, G, P = 64, 2, 32
    c = Cache(1, pages_for([n], P), P, -(-n // P), 1, 1, d).fill([n], shuffle=1)
    v = bf16((1, 1, 1, n, d), 4).double().clamp(-3, 3)
    v[..., :n // 2, :] *= before
    v[..., n // 2:, :] *= after
    R.kv_append_q4(c.pool, c.pages, bf16((1, 1, 1, n, d), 3).to(DEV), v.bfloat16().to(DEV), i32([0]))
    c.want = c.pool.cpu().numpy()
    q = bf16((1, 1, G, d), 9)
    out = torch.empty((1, 1, G, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


@pytest.mark.parametrize("n", [300, 4000])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 16, 2.0 ** 40])
@pytest.mark.parametrize("scale", [20.0, 2.0 ** 30])
def test_attention_of_large_equal_logits(n, size, scale):
    """Keys that are all the same, with logits of 2^27 and more, whose steps in
    fp32 are larger than any exponent of two that the values' size asks for: the
    mean of the values.  Equal logits give equal probabilities, so an output is
    off by n rounded additions and, 22 bits of each product, 2^-21 of mean |v|."""
    d, G, P = 128, 3, 32
    c = Cache(1, pages_for([n], P), P, -(-n // P), 1, 1, d).fill([n], shuffle=1)
    k = torch.full((1, 1, 1, n, d), 2896.0 * size / 4096)
    v = bf16((1, 1, 1, n, d), 4).clamp(-1, 1) * scale
    R.kv_append_q4(c.pool, c.pages, k.bfloat16().to(DEV), v.to(DEV), i32([0]))
    c.want = c.pool.cpu().numpy()
    q = torch.full((1, 1, G, d), size).bfloat16()
    out = torch.empty((1, 1, G, d), device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    v64 = c.rows(0, 0, 0)[1]
    tol = ((n + 64) * 2.0 ** -24 + 2.0 ** -20) * np.abs(v64).mean(0)
    assert (np.abs(f64(out)[0, 0] - v64.mean(0)) <= tol).all()


@pytest.mark.parametrize("n", [130, 2000])
@pytest.mark.parametrize("q0, k0", [(1.0, 2.0 ** 104), (2.0 ** -20, 2.0 ** 104), (2.0 ** 20, 2.0 ** 98),
                                    (2.0 ** 100, 2.0 ** 18), (2.0 ** 127, 2.0 ** -9)])
def test_attention_of_the_largest_keys_and_queries(n, q0, k0):
    """Keys up to the header's limit, and queries up to bf16's, of logits up to
    2^122: the row of the largest has all the weight.  d 128, so that all four
    groups add up."""
    d, P = 128, 32
    c = Cache(1, pages_for([n], P), P, -(-n // P), 1, 1, d).fill([n], shuffle=1)
    k = torch.full((1, 1, 1, n, d), k0)
    best = n // 3
    k[..., best, :] *= 1.5
    k[..., ::5, :] *= -1.0
    k[..., best, :] = k[..., best, :].abs()
    R.kv_append_q4(c.pool, c.pages, k.bfloat16().to(DEV), bf16((1, 1, 1, n, d), 4).to(DEV), i32([0]))
    c.want = c.pool.cpu().numpy()
    q = torch.full((1, 1, 3, d), q0)
    q[0, 0, 1] *= -1.0                                        # (the rows of the least: equal logits, not checked)
    q[0, 0, 2] = 0.0
    out = torch.empty((1, 1, 3, d), device=DEV)
    R.decode_attention_q4(q.bfloat16().to(DEV), c.pool, c.pages, out)
    got, v = f64(out)[0, 0], c.rows(0, 0, 0)[1]
    assert np.isfinite(got).all()
    assert (np.abs(got[0] - v[best]) <= 2.0 ** -20 * np.abs(v[best])).all()
    assert (np.abs(got[2] - v.mean(0)) <= ((n + 64) * 2.0 ** -24 + 2.0 ** -20) * np.abs(v).mean(0)).all()


@pytest.mark.parametrize("n", [40, 1000])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_query_that_is_not_finite_over_empty_slots(n, bad):
    """It reaches no row of a sequence of empty slots, whose outputs are zeros;
    where there are rows it gives NaN, and the other heads keep their outputs."""
    d, P, G = 64, 16, 3
    lens = [n, n, 0, n]
    c = Cache(4, pages_for(lens, P), P, -(-n // P), 1, 1, d).fill(lens, shuffle=1)
    batch = R.Batch(1, 4, G, 1, d, n)
    k, v = bf16((1, 4, 1, n, d), 1).to(DEV), bf16((1, 4, 1, n, d), 2).to(DEV)
    idx = torch.arange(n, dtype=torch.int32).repeat(4, 1).view(1, 4, 1, n)
    idx[:, 1] = -1
    idx[:, 3, :, 3:] = -1
    R.kv_compact_q4(batch, k, v, idx.to(DEV), 1.0, c.pool, c.pages, i32([0, 0, -1, 0]))
    c.want = c.pool.cpu().numpy()
    q = bf16((1, 4, G, d), 9)
    q[:, :, 1, 5] = bad
    out = torch.full((1, 4, G, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    got = out.cpu()
    assert torch.isnan(got[0, 0, 1]).all() and torch.isnan(got[0, 3, 1]).all()
    assert (got[0, 1:3] == 0).all()
    q[:, :, 1, 5] = 0
    want = torch.empty_like(out)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, want)
    out[:, :, 1] = want[:, :, 1]
    check_attention(out, q, c)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("budget", [0.1, 0.9])
def test_compact_from_pinned_host_memory(budget, packed):
    """K and V left in pinned host memory, a few rows and whole records: the
    bytes that the same rows on the device give."""
    L, b, Hkv, n, d, P = 2, 2, 2, 40, 128, 16
    shape = (L, b * n, Hkv, d) if packed else (L, b, Hkv, n, d)
    k, v = bf16(shape, 1), bf16(shape, 2)
    batch = R.Batch(L, b, Hkv, Hkv, d, n, seqlens=[n, n] if packed else None)
    m = R.kept_rows(n, budget)
    idx = torch.sort(torch.rand((L, b, Hkv, n), generator=torch.Generator().manual_seed(3)).topk(m).indices).values
    idx = idx.permute(0, 2, 1, 3).reshape(L, Hkv, b * m) if packed else idx
    lens = [m + 3] * b
    pools = []
    for where in ("device", "host", "one each"):
        c = Cache(b, pages_for(lens, P), P, 4, L, Hkv, d, seed=1).fill(lens, shuffle=1)
        kk = k.to(DEV) if where == "device" else k.pin_memory()
        vv = v.pin_memory() if where == "host" else v.to(DEV)
        st = new_status()
        R.kv_compact_q4(batch, kk, vv, idx.int().contiguous().to(DEV), budget, c.pool, c.pages, i32([3] * b), status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
        pools.append(c.pool.cpu())
    assert torch.equal(pools[0], pools[1]) and torch.equal(pools[0], pools[2])
    for kk, vv in ((k, v.to(DEV)), (k.to(DEV), v), (k, v)):
        with pytest.raises(ValueError, match="pinned"):
            R.kv_compact_q4(batch, kk, vv, idx.int().contiguous().to(DEV), budget, c.pool, c.pages, i32([3] * b))
    with pytest.raises(ValueError, match="current device"):
        R.kv_append_q4(c.pool, c.pages, bf16((L, b, Hkv, 1, d), 1).pin_memory(), bf16((L, b, Hkv, 1, d), 2).to(DEV),
                       i32([3] * b))


@pytest.mark.parametrize("entry", [-1, 1 << 20])
def test_rows_without_a_page_are_not_read_back(entry):
    """A table entry that names no page: its rows are absent, and their outputs
    stay as they were."""
    d, P, n = 64, 16, 50
    c = Cache(1, 6, P, 4, 1, 2, d).fill([n], shuffle=4).random_rows(3)
    c.pages.table[0, 1] = entry
    out = [torch.full((1, 1, 2, n, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    st = new_status()
    R.kv_expand_q4(c.pool, c.pages, *out, status=st)
    assert st.item() == R.STATUS_BAD_INDEX
    for h in range(2):
        for o, want in zip(out, c.rows(0, 0, h)):
            want = torch.from_numpy(want).float().bfloat16()
            want[P:2 * P] = 7.0
            assert torch.equal(o[0, 0, h].cpu(), want)


def test_a_book_of_more_slots_than_a_batch_takes():
    """Tens of thousands of slots of a pool of many layers and heads, a few of
    them in use: room made, pages shared and copied, pages moved."""
    L, Hkv, d, P, n_seqs = 32, 8, 64, 16, 20000
    c = Cache(n_seqs, 12, P, 2, L, Hkv, d, seed=1)
    use = [3, 1500, 19999]
    for i, s in enumerate(use):
        c.book.lens[s], c.book.table[s][0], c.book.refs[2 * i + 4] = 7 + i, 2 * i + 4, 1
    c.upload()
    parent = list(range(n_seqs))
    parent[17000] = 1500
    c.book.fork(parent)
    R.kv_pages_fork(c.pages, i32(parent))
    c.check_book()
    add, pos, st = [0] * n_seqs, torch.full((n_seqs,), 9, dtype=torch.int32, device=DEV), new_status()
    for s in (3, 1500, 17000):
        add[s] = 10
    R.kv_pages_reserve(c.pages, c.pool, i32(add), pos, status=st)
    want, copies = c.book.reserve(add)
    for src, dst, rows in copies:
        recs = -(-rows // 16)
        c.want[:, dst, :, :recs] = c.want[:, src, :, :recs]
    assert pos.tolist() == want and st.item() == 0
    c.check_book()
    c.check_pool()
    live = torch.zeros(1, dtype=torch.int32, device=DEV)
    R.kv_pages_pack(c.pages, c.pool, n_live=live)
    n, moves = c.book.pack()
    for src, dst in moves:
        c.want[:, dst] = c.want[:, src]
    assert live.item() == n and len(moves) > 0
    c.check_book()
    got = c.pool.cpu().numpy()
    assert np.array_equal(got[:, :n], c.want[:, :n])


@pytest.mark.parametrize("more", [0, 1])
def test_attention_around_the_choice_of_join_on_this_device(more):
    """As many units as are joined one by one, a unit to four CTAs, and one more."""
    d, P, n = 64, 64, 900
    units = 3 * sms() // 4 + more
    c = Cache(units, units * 15, P, 15, 1, 1, d).fill([n if s % 7 else 0 for s in range(units)], shuffle=2)
    k, v = (bf16((1, units, 1, n, d), x).to(DEV) for x in (1, 2))
    R.kv_append_q4(c.pool, c.pages, k, v, i32([0 if s % 7 else -1 for s in range(units)]))
    c.want = c.pool.cpu().numpy()
    q = bf16((1, units, 2, d), 9)
    out = torch.full((1, units, 2, d), 7.0, device=DEV)
    R.decode_attention_q4(q.to(DEV), c.pool, c.pages, out)
    check_attention(out, q, c)


def store_waves(units, items):
    """Waves of the SMs' 32 warps that a call of so many items has."""
    return units * items / (32 * sms())


def kept_of(rng, n, m):
    """m ascending positions of n tokens, every eighth an empty slot."""
    x = np.sort(rng.permutation(n)[:m])
    x[rng.random(x.size) < 0.125] = -1
    return x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("above", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_compact_around_the_choice_of_items_a_warp(d, above, packed):
    """Calls just below and from so many warps on that each takes several items
    one after another (six waves of them): every row's bytes, and nothing else,
    at every place in a record, with items that are no multiple of a warp's, and
    in the packed batch with sequences without tokens and of very different
    lengths."""
    Hkv, L, P, budget = 4, 1, 48, 0.5
    rng = np.random.default_rng(d + above)
    if packed:
        lens = [0, 1, 1200, 3] + [int(x) for x in rng.integers(0, 60, 12)]
    else:
        lens = [36]
    top = R.kept_rows(max(lens), budget)
    items = ((top + 14) // 16 + 1) * (2 if d == 128 else 1)
    assert packed or items % 4 != 0
    b = -(-6 * 32 * sms() // (items * Hkv)) - (0 if above else 1)
    assert (store_waves(b * Hkv, items) >= 6) == above
    if packed:
        lens += [int(x) for x in rng.integers(0, 60, b - len(lens))]
    else:
        lens = lens * b
    assert len(lens) == b
    kept = [R.kept_rows(n, budget) for n in lens]
    pos = [int(x) for x in rng.integers(0, 40, b)]
    pos[0:3] = [0, 15, 8]
    rows = [p + m for p, m in zip(pos, kept)]
    c = Cache(b, pages_for(rows, P), P, -(-max(rows) // P), L, Hkv, d, seed=1).fill(rows, shuffle=3)
    T = sum(lens)
    k, v = bf16((L, T, Hkv, d), 1), bf16((L, T, Hkv, d), 2, 3.0)      # (token rows, also of the dense batch)
    batch = R.Batch(L, b, Hkv, Hkv, d, max(lens), seqlens=lens if packed else None)
    if packed:
        kd, vd = k.to(DEV), v.to(DEV)
    else:
        kd, vd = (x.view(L, b, 36, Hkv, d).transpose(2, 3).to(DEV) for x in (k, v))
    at = np.cumsum([0] + lens)
    idx = [[kept_of(rng, n, m) for n, m in zip(lens, kept)] for _ in range(Hkv)]
    if packed:
        keep = np.stack([np.concatenate(x) for x in idx])[None]
    else:
        keep = np.stack([np.stack(x) for x in idx], 1)[None]          # [L][b][Hkv][K]
    k64, v64 = f64(k)[0], f64(v)[0]
    for h in range(Hkv):
        j = np.concatenate([np.arange(m) for m in kept])
        s = np.repeat(np.arange(b), kept)
        t = np.concatenate(idx[h])
        token = at[s] + np.maximum(t, 0)
        row = np.asarray(pos)[s] + j
        page = np.asarray(c.book.table)[s, row // P]
        recs = c.want[0].reshape(-1, 18 * d)
        Q.write_rows(recs, (page * Hkv + h) * (P // 16) + row % P // 16, row % 16, k64[token, h], v64[token, h], t < 0)
    st = new_status()
    R.kv_compact_q4(batch, kd, vd, torch.from_numpy(keep).int().to(DEV), budget, c.pool, c.pages, i32(pos), status=st)
    c.check_pool()
    assert st.item() == 0


@pytest.mark.parametrize("form", ["rows", "rows of four heads", "records"])
def test_every_mantissa_and_group_maximum(form):
    """Every 8-bit mantissa of an element with every one of its group's largest
    element, at each exponent that gives a code of its own, both signs, half-way
    quotients among them, and at scales about 2^-126 and of the largest: the
    oracle's bytes from each of the storing kernels."""
    d = 128
    rows = []
    for e in (0, 120, -131):
        m = np.arange(128, 256)
        x = np.concatenate([np.ldexp(np.arange(128.0, 256.0), -i) for i in range(7)])  # 896 for each maximum
        x = np.concatenate([x, np.zeros(-x.size % 31)]).reshape(-1, 31)
        g = np.concatenate([np.broadcast_to(m[:, None, None], (128, x.shape[0], 1)),
                            np.broadcast_to(x[None], (128,) + x.shape)], -1)
        g = np.where(np.abs(g) <= g[..., :1], g, 0.0).reshape(-1, 32)
        g[1::2] *= -1.0
        rows.append(np.ldexp(g[:g.shape[0] // 4 * 4].reshape(-1, d), e))
    x = torch.from_numpy(np.concatenate(rows)).bfloat16()
    n = x.shape[0]
    k, v = f64(x), f64(x.flip(1))
    vd = x.flip(1)
    if form == "records":
        P = 1024
        c = Cache(1, -(-n // P), P, -(-n // P), 1, 1, d).fill([n])
        R.kv_append_q4(c.pool, c.pages, x.to(DEV).view(1, 1, 1, n, d), vd.to(DEV).view(1, 1, 1, n, d), i32([0]))
        page, row, heads = np.arange(n) // P, np.arange(n) % P, 1
    else:
        P, heads = 16, 1 if form == "rows" else 4
        L = 1 if heads == 1 else -(-2 * 32 * sms() // (n * heads))
        assert (store_waves(L * n * heads, 1) >= 2) == (heads > 1)
        c = Cache(n, n, P, 1, L, heads, d).fill([16] * n)
        kd, vv = (y.to(DEV).view(1, n, 1, 1, d).expand(L, n, heads, 1, d).contiguous() for y in (x, vd))
        R.kv_append_q4(c.pool, c.pages, kd, vv, i32([s % 16 for s in range(n)]))
        page, row = np.arange(n), np.arange(n) % 16
    for l in range(c.want.shape[0]):
        for h in range(heads):
            recs = c.want[l].reshape(-1, 18 * d)
            Q.write_rows(recs, (page * heads + h) * (P // 16) + row // 16, row % 16, k, v)
    c.check_pool()
