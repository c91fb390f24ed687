"""The paged cache's operators against their float64 oracle: every output and
every slot of the pool, through PagedCache (and so through the C ABI).

Bounds (none is fitted).  u = eps / 2 of the 16-bit type is the most that one
rounding moves a value, relative to it.
 Append: a norm's sum of dh squares, its root and products are off by at most
 (dh + 8) 2^-24 of a value; sine and cosine by 2^-21 (an angle reduced in double
 and rounded to fp32 within half a turn: 2^-24 turns = 2^-21 rad, and the
 functions' own few 2^-24); one rounding at the end.
 Attention: a score is off by (dh + 8) 2^-23 of scale sum |q_i k_i|, so a
 probability by that much of itself (twice: its share of the sum too), the
 exponential and the sums over n slots by (n + 64) 2^-23; each probability is
 rounded once to 16 bits (u), all of it in units of sum p |v|; the output is
 rounded once (u).  fp16 adds its smallest step: 2^-25 in an output, and in a
 probability 2^-25 / 2^6 of at least the largest probability, n of them.
"""
import numpy as np
import pytest
import torch

from oracle import paged as op

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _np(t):
    return t.detach().to("cpu", torch.float64).numpy()


def _u(t):
    return torch.finfo(TYPES[t]).eps / 2


def _tiny(t):
    return 2.0 ** -25 if t == "fp16" else 0.0


class Pool:
    """A pool whose pages lie in a shuffled order, table entries past a
    sequence's pages hold numbers of no page, and every slot that no sequence
    holds is NaN."""

    def __init__(self, seed, t, kv, dh, page, lengths, spare=2, extra_columns=2):
        from paper_2608_10824_amd.paged import PagedCache
        self.r = r = np.random.default_rng(seed)
        self.t, self.kv, self.dh, self.page, self.lengths = t, kv, dh, page, list(lengths)
        used = [-(-n // page) for n in lengths]
        n_pages = sum(used) + spare
        columns = max(used) + extra_columns
        ids = r.permutation(n_pages)
        self.table = r.choice(np.array([-1, n_pages, 2 ** 31 - 1, -2 ** 31]), (len(lengths), columns)).astype(np.int32)
        at = 0
        for s, n in enumerate(used):
            self.table[s, :n] = ids[at:at + n]
            at += n
        k = np.full((n_pages, kv, page, dh), np.nan)
        v = np.full((n_pages, kv, dh, page), np.nan)
        for s, n in enumerate(lengths):
            for j in range(n):
                p, o = self.table[s, j // page], j % page
                k[p, :, o], v[p, :, :, o] = r.standard_normal((kv, dh)), r.standard_normal((kv, dh))
        self.cache = PagedCache(torch.tensor(k).to(TYPES[t]).to(DEV), torch.tensor(v).to(TYPES[t]).to(DEV),
                                torch.tensor(self.table, device=DEV))

    def rows(self, n, heads, scale=1.0):
        return torch.tensor(self.r.standard_normal((n, heads, self.dh)) * scale).to(TYPES[self.t]).to(DEV)

    def ints(self, x):
        return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)

    def expect(self, out, q, seqs, lasts, window=0, sinks=0, scale=None):
        """Compares attention outputs with the oracle's, row by row."""
        k, v, q, out = _np(self.cache.k_pages), _np(self.cache.v_pages), _np(q), _np(out)
        scale = self.dh ** -0.5 if scale is None else scale
        u, worst = _u(self.t), 0.0
        for r, (s, last) in enumerate(zip(seqs, lasts)):
            want, mag, top, n = op.attend_row(q[r], s, last, k, v, self.table, scale, window, sinks)
            if n == 0:
                assert not out[r].any(), "row %d sees nothing and is not zero" % r
                continue
            p = (2 * (self.dh + 8) * 2.0 ** -23 * top + (n + 64) * 2.0 ** -23 + u)[:, None]
            vmax = np.nanmax(np.abs(np.where(np.isfinite(v), v, 0)))
            tol = u * np.abs(want) + mag * p * (1 + u) + _tiny(self.t) * (1 + n / 64 * vmax)
            assert np.array_equal(np.isnan(out[r]), np.isnan(want)), "row %d: NaN" % r
            fine = np.isfinite(want)
            assert np.array_equal(out[r][~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), "row %d: inf" % r
            off = (np.abs(out[r] - want) / tol)[fine]
            assert off.size == 0 or off.max() <= 1, "row %d (sequence %d, last %d): %.3g of the bound" % (r, s, last, off.max())
            worst = max([worst] + list(off[:1]))
        return worst


# ------------------------------------------------------------------- append
def _append(seed, t, heads, kv, dh, page, lengths, rows, pairs=None, positions=None, norm=False, fused=True,
            theta=1e4, eps=1e-5, with_q=True, q_out=None):
    """Appends rows (sequence, slot) and checks q_out and the whole pool."""
    pool = Pool(seed, t, kv, dh, page, lengths)
    n, r = len(rows), pool.r
    if fused:
        x = pool.rows(n, heads + 2 * kv)
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    else:
        q, k, v = pool.rows(n, heads), pool.rows(n, kv), pool.rows(n, kv)
    gains = [torch.tensor(1 + 0.2 * r.standard_normal(dh)).to(TYPES[t]).to(DEV) if norm else None for _ in range(2)]
    c = pool.cache
    before_k, before_v = c.k_pages.clone(), c.v_pages.clone()
    pos = None if positions is None else pool.ints(positions).reshape(-1, n)
    got = c.append(q if with_q else None, k, v, pool.ints([s for s, _ in rows]), pool.ints([j for _, j in rows]),
                   positions=pos, rope_pairs=pairs, rope_theta=theta, q_norm=gains[0], k_norm=gains[1], rms_eps=eps,
                   q_out=q_out)
    want_pairs = (dh // 2,) if pairs is None else pairs
    u = _u(t)

    def expect(out, x, row, gain):
        p = [rows[row][1]] * 3 if positions is None else [positions[a][row] for a in range(len(want_pairs))]
        for h in range(x.shape[0]):
            normed = x[h] / np.sqrt(np.mean(x[h] ** 2) + eps) * gain if gain is not None else x[h]
            want = op.rope_norm(x[h], p, want_pairs, theta, gain, eps)
            m = sum(want_pairs)
            mag = np.abs(normed)
            mag[:2 * m] = np.tile(mag[:m] + mag[m:2 * m], 2)
            tol = u * np.abs(want) + mag * (2.0 ** -20 + (dh + 8) * 2.0 ** -24) * (1 + u) + _tiny(t)
            assert (np.abs(out[h] - want) <= tol).all(), "row %d head %d: %.3g of the bound" % (
                row, h, (np.abs(out[h] - want) / tol).max())

    qn, kn, vn = _np(q), _np(k), _np(v)
    gq, gk = [None if g is None else _np(g) for g in gains]
    if with_q:
        assert got.shape == q.shape
        o = _np(got)
        for i in range(n):
            expect(o[i], qn[i], i, gq)
    else:
        assert got is None
    ko, vo = _np(c.k_pages), _np(c.v_pages)
    for i, (s, j) in enumerate(rows):
        at = op.place(pool.table, c.k_pages.shape[0], page, s, j)
        if at is None:
            continue
        expect(ko[at[0], :, at[1]], kn[i], i, gk)
        assert np.array_equal(vo[at[0], :, :, at[1]], vn[i])
        # put the slot back: what remains has to be as it was, bit for bit
        c.k_pages[at[0], :, at[1]] = before_k[at[0], :, at[1]]
        c.v_pages[at[0], :, :, at[1]] = before_v[at[0], :, :, at[1]]
    assert torch.equal(c.k_pages.view(torch.int16), before_k.view(torch.int16))
    assert torch.equal(c.v_pages.view(torch.int16), before_v.view(torch.int16))
    return pool


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,dh,page", [(8, 2, 128, 16), (4, 4, 64, 32), (7, 1, 128, 64), (6, 3, 64, 128), (1, 1, 64, 16)])
def test_append_rows_of_a_prompt(t, heads, kv, dh, page):
    """Rows of three sequences: a prompt from slot 0, one row, a run that starts
    and ends inside a page and skips slots; norm and one axis."""
    rows = [(0, j) for j in range(70)] + [(1, 5)] + [(2, j) for j in range(13, 61) if j % 7 != 3]
    _append(1, t, heads, kv, dh, page, [70, 20, 61], rows, norm=True)


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("dh,pairs", [(128, (16, 24, 24)), (128, (8, 12, 12)), (64, (5, 3)), (64, (0, 7, 1)), (128, ()),
                                      (128, (4,)), (64, (3, 1, 28))])
def test_append_axes_and_partial_rotation(t, dh, pairs):
    n = 37
    rows = [(0, j) for j in range(n)]
    positions = [[(j * 7 + a * 1000) % 977 - 100 * a for j in range(n)] for a in range(len(pairs))] if pairs else None
    _append(2, t, 3, 1, dh, 16, [40], rows, pairs=pairs, positions=positions, norm=dh == 64, fused=False)


def test_append_far_positions():
    """Positions to the end of int32, a long base: the angle keeps its fraction of a turn."""
    n = 9
    far = [0, 1, 10 ** 5, 10 ** 6 + 1, 10 ** 7 + 3, 123456789, 2 ** 31 - 1, -1, -2 ** 31]
    _append(3, "fp16", 2, 2, 128, 16, [n], [(0, j) for j in range(n)], positions=[far], pairs=(64,), theta=1e6)


@pytest.mark.parametrize("theta", [10000 * 8 ** (128 / 126), 1234567.89, 0.7])
def test_append_far_positions_of_bases_that_fp32_does_not_hold(theta):
    far = [0, 1, 10 ** 5, 10 ** 7 + 3, 123456789, 2 ** 31 - 1, -2 ** 31]
    n = len(far)
    _append(67, "fp16", 2, 2, 128, 16, [n], [(0, j) for j in range(n)], positions=[far], pairs=(64,), theta=theta)


def test_append_rows_in_any_order_of_any_run_length():
    r = np.random.default_rng(4)
    every = [(s, j) for s, n in enumerate([50, 33, 0, 129]) for j in range(n)]
    for n in (1, 2, 15, 63, 64, 65, 150):
        _append(5 + n, "bf16", 4, 2, 64, 16, [50, 33, 0, 129], [every[i] for i in r.permutation(len(every))[:n]])


@pytest.mark.parametrize("first", range(0, 17, 3))
def test_append_runs_at_any_offset(first):
    _append(40 + first, "fp16", 2, 2, 128, 32, [400], [(0, first + j) for j in range(300)], fused=False)


def test_append_skips_rows_without_a_place():
    """Padding rows (sequence -1), slots past the table, pages that do not exist:
    no slot changes, q comes all the same."""
    rows = [(0, 0), (-1, 0), (0, 1), (3, 0), (2 ** 30, 5), (0, -1), (0, 16 * 20), (0, 17), (1, 3), (1, 40), (-2 ** 31, 2 ** 31 - 1)]
    _append(6, "bf16", 4, 2, 128, 16, [20, 33, 1], rows, norm=True)


def test_append_without_queries_and_into_a_given_tensor():
    rows = [(0, j) for j in range(20)]
    _append(7, "bf16", 4, 2, 128, 16, [20], rows, with_q=False)
    whole = torch.full((20, 6, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    _append(8, "bf16", 4, 2, 128, 16, [20], rows, q_out=whole[:, 1:5])
    assert (whole[:, 0] == 9).all() and (whole[:, 5] == 9).all()


def test_append_nothing():
    pool = Pool(9, "bf16", 2, 64, 16, [5])
    q = pool.cache.append(pool.rows(0, 4), pool.rows(0, 2), pool.rows(0, 2), pool.ints([]), pool.ints([]))
    assert q.shape == (0, 4, 64)


# ------------------------------------------------------------------- decode
LENGTHS = [1, 0, 15, 16, 17, 31, 32, 33, 200, 129, 64]


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,dh,page", [(4, 4, 128, 16), (8, 2, 128, 32), (14, 2, 64, 16), (16, 1, 128, 128),
                                              (40, 1, 64, 64), (34, 2, 128, 16)])
def test_decode_lengths(t, heads, kv, dh, page):
    """One to hundreds of slots, an idle sequence, groups of one to forty query
    heads; stale NaN behind every sequence's end."""
    pool = Pool(11, t, kv, dh, page, LENGTHS)
    q = pool.rows(len(LENGTHS), heads, 2.0)
    out = pool.cache.decode(q, pool.ints(LENGTHS))
    pool.expect(out, q, range(len(LENGTHS)), [n - 1 for n in LENGTHS])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 0), (33, 40), (100, 4), (100, 64), (199, 1), (200, 7), (2 ** 31 - 1, 5), (7, 2 ** 31 - 1)])
def test_decode_window_and_sinks(window, sinks):
    pool = Pool(12, "bf16", 2, 64, 16, LENGTHS + [333])
    n = len(LENGTHS) + 1
    q = pool.rows(n, 6, 2.0)
    out = pool.cache.decode(q, pool.ints(LENGTHS + [333]), window=window, sinks=sinks)
    pool.expect(out, q, range(n), [m - 1 for m in LENGTHS + [333]], window, sinks)


@pytest.mark.parametrize("t,dh,page", [("bf16", 128, 16), ("fp16", 64, 64), ("fp16", 128, 128)])
def test_decode_one_long_sequence(t, dh, page):
    """A few rows over thousands of slots (split over the length and joined), beside short ones."""
    lengths = [5000, 3, 1, 2777]
    pool = Pool(13, t, 2, dh, page, lengths)
    q = pool.rows(4, 8, 2.0)
    out = pool.cache.decode(q, pool.ints(lengths))
    pool.expect(out, q, range(4), [n - 1 for n in lengths])
    out = pool.cache.decode(q, pool.ints(lengths), window=2500, sinks=70)
    pool.expect(out, q, range(4), [n - 1 for n in lengths], 2500, 70)


def test_decode_strides_scale_and_out():
    pool = Pool(14, "fp16", 2, 64, 16, [40, 77])
    wide = pool.rows(2, 9)
    q = wide[:, 2:8]
    held = torch.full((2, 8, 64), 3.0, dtype=torch.float16, device=DEV)
    out = pool.cache.decode(q, pool.ints([40, 77]), scale=0.3, out=held[:, 1:7])
    assert out.data_ptr() == held[:, 1:7].data_ptr() and (held[:, 0] == 3).all() and (held[:, 7] == 3).all()
    pool.expect(out, q, [0, 1], [39, 76], scale=0.3)


def test_decode_steep_scores():
    """Scores over hundreds: the running maximum moves tile by tile, up and down."""
    pool = Pool(15, "bf16", 1, 128, 16, [700, 700])
    c = pool.cache
    for s in range(2):
        for j in range(700):
            p = pool.table[s, j // 16]
            c.k_pages[p, 0, j % 16] *= (j if s == 0 else 700 - j) / 100
    q = pool.rows(2, 4, 4.0)
    pool.expect(c.decode(q, pool.ints([700, 700])), q, [0, 1], [699, 699])


def test_decode_lengths_past_the_table_and_below_zero():
    """A length over what the table holds ends at the table's last slot; a negative one is an idle slot."""
    pool = Pool(16, "bf16", 2, 64, 16, [48, 48, 30], extra_columns=0)
    q = pool.rows(3, 4)
    out = pool.cache.decode(q, pool.ints([2 ** 31 - 1, 49, -2 ** 31]))
    pool.expect(out, q, range(3), [47, 47, -1])


def test_pages_that_do_not_exist_are_not_seen():
    pool = Pool(17, "bf16", 2, 64, 16, [90, 40, 16, 20])
    c = pool.cache
    for s, col, to in ((0, 0, -1), (0, 3, c.k_pages.shape[0]), (1, 2, 2 ** 31 - 1), (2, 0, -7)):
        pool.table[s, col] = to
    c.page_table.copy_(torch.tensor(pool.table))
    q = pool.rows(4, 4)
    out = c.decode(q, pool.ints([90, 40, 16, 20]))
    pool.expect(out, q, range(4), [89, 39, 15, 19])
    assert not out[2].any()
    q = pool.rows(8, 4)
    lasts = [5, 15, 20, 89, 39, 0, 15, 19]
    out = c.prefill(q, pool.ints(lasts), pool.ints([0, 4, 5, 7, 8]))
    pool.expect(out, q, [0, 0, 0, 0, 1, 2, 2, 3], lasts)


def test_infinities_and_nan_in_sight():
    """What a row sees comes through; a score of -inf everywhere is 0/0."""
    pool = Pool(18, "bf16", 1, 64, 16, [40, 40, 40, 40])
    c, t = pool.cache, pool.table
    c.v_pages[t[0, 1], 0, 3, 4] = float("inf")
    c.v_pages[t[1, 2], 0, 5, 1] = float("nan")
    c.k_pages[t[2, 0], 0, 7, 0] = float("nan")
    q = pool.rows(4, 2)
    out = c.decode(q, pool.ints([40] * 4))
    assert torch.isinf(out[0, :, 3]).all() and torch.isnan(out[1, :, 5]).all() and torch.isnan(out[2]).all()
    pool.expect(out, q, range(4), [39] * 4)
    for s in (3,):
        for col in range(3):
            c.k_pages[t[s, col], 0, :, 0] = float("inf")
    q[3, :, 0] = -1.0
    assert torch.isnan(c.decode(q, pool.ints([40] * 4))[3]).all()


# ------------------------------------------------------------------ prefill
def _ragged(pool, heads, per_seq, window=0, sinks=0, lasts=None, scale=2.0):
    """Prefill of per_seq[s] = the last slots of sequence s's rows."""
    flat = [j for rows in per_seq for j in rows]
    seqs = [s for s, rows in enumerate(per_seq) for _ in rows]
    begin = np.concatenate([[0], np.cumsum([len(x) for x in per_seq])])
    q = pool.rows(len(flat), heads, scale)
    out = pool.cache.prefill(q, pool.ints(flat), pool.ints(begin), window=window, sinks=sinks)
    pool.expect(out, q, seqs, flat, window, sinks)
    return q, out, seqs, flat, begin


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,dh,page", [(4, 4, 128, 16), (8, 2, 128, 64), (14, 2, 64, 16), (3, 1, 128, 128), (40, 1, 64, 32)])
def test_prefill_ragged(t, heads, kv, dh, page):
    """Whole prompts, one row, no row, chunks behind a cached prefix, rows with gaps, rows in falling order."""
    pool = Pool(21, t, kv, dh, page, [150, 1, 40, 260, 97, 66])
    r = pool.r
    gaps = sorted(r.permutation(97)[:41])
    _ragged(pool, heads, [range(150), [0], [], range(201, 260), gaps, range(65, -1, -1)])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (9, 4), (64, 0), (31, 33), (130, 5), (64, 200), (300, 2)])
def test_prefill_window_and_sinks(window, sinks):
    pool = Pool(22, "bf16", 1, 64, 16, [333, 20, 180])
    _ragged(pool, 3, [range(140, 333), range(20), range(0, 180, 3)], window, sinks)


def test_prefill_few_rows_over_many_slots():
    pool = Pool(23, "bf16", 2, 128, 64, [4000, 2500])
    _ragged(pool, 4, [range(3990, 4000), [2499]])
    _ragged(pool, 4, [[3999, 10, 2000], [2499, 0]], 1500, 70)
    pool = Pool(24, "fp16", 1, 64, 16, [3001])
    _ragged(pool, 2, [range(2900, 3001)])


def test_prefill_block_that_sees_both_ways():
    """Rows of an action block give the block's last slot: they see each other."""
    pool = Pool(25, "bf16", 2, 64, 16, [100])
    _ragged(pool, 4, [list(range(80)) + [99] * 20])


def test_prefill_rows_that_see_nothing_and_rows_of_no_sequence():
    pool = Pool(26, "bf16", 2, 64, 16, [50, 50, 50])
    lasts = [-1, 3, -1, 49, -5, -1, -1, 7, 8, 9]
    q = pool.rows(10, 4)
    held = torch.full((10, 4, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints([1, 4, 7, 8]), out=held)
    assert (held[0] == 5).all() and (held[8:] == 5).all()
    pool.expect(out[1:8], q[1:8], [0, 0, 0, 1, 1, 1, 2], lasts[1:8])
    # bounds that do not rise, or pass the rows, cover what lies inside
    held.fill_(5.0)
    out = pool.cache.prefill(q, pool.ints([9] * 10), pool.ints([4, 2, 5, 99]), out=held)
    assert (held[:2] == 5).all() and not (held[2:] == 5).any()
    pool.expect(out[2:], q[2:], [1] * 3 + [2] * 5, [9] * 8)


@pytest.mark.parametrize("rows,length", [(10, 50), (10, 3000), (300, 3000), (400, 3000)])
def test_prefill_with_bounds_that_fall(rows, length):
    """Bounds have to rise; where they do not, no row outside them is touched (nor any other memory)."""
    pool = Pool(26, "bf16", 2, 64, 16, [length] * 4)
    q = pool.rows(rows + 9, 4)
    held = torch.full((rows + 9, 4, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    pool.cache.prefill(q, pool.ints([length - 1] * (rows + 9)), pool.ints([0, rows, 0, rows, rows + 7]), out=held)
    assert (held[rows + 7:] == 5).all()


def test_values_of_later_slots_do_not_reach_earlier_rows():
    """NaN and infinities in the keys and values of slots that only later rows
    see: earlier rows are finite and right, later ones show them."""
    for window, sinks in ((0, 0), (40, 4)):
        pool = Pool(27, "bf16", 2, 64, 16, [200])
        c, t = pool.cache, pool.table
        c.v_pages[t[0, 5], 0, 3, 7] = float("nan")    # slot 87
        c.v_pages[t[0, 8], 1, 9, 1] = float("inf")    # slot 129
        c.k_pages[t[0, 9], 0, 15, 0] = float("nan")   # slot 159
        q, out, seqs, flat, begin = _ragged(pool, 4, [range(200)], window, sinks)
        o = _np(out)
        assert np.isfinite(o[:87]).all() and np.isnan(o[87, :2, 3]).all() and np.isfinite(o[:159, 2:, :9]).all()
        assert np.isinf(o[129, 2:, 9]).all() and np.isnan(o[159, :2]).all()
        if window:
            assert np.isfinite(o[199]).all()


def test_prefill_steep_scores():
    pool = Pool(28, "fp16", 1, 64, 16, [300])
    for j in range(300):
        pool.cache.k_pages[pool.table[0, j // 16], 0, j % 16] *= (j % 50) / 10
    _ragged(pool, 4, [range(300)], scale=4.0)


def test_prefill_of_one_row_is_decode():
    pool = Pool(29, "bf16", 2, 128, 16, [37, 600, 1])
    q = pool.rows(3, 8)
    d = pool.cache.decode(q, pool.ints([37, 600, 1]))
    p = pool.cache.prefill(q, pool.ints([36, 599, 0]), pool.ints([0, 1, 2, 3]))
    pool.expect(d, q, range(3), [36, 599, 0])
    pool.expect(p, q, range(3), [36, 599, 0])


@pytest.mark.parametrize("seqs,heads,kv", [(64, 4, 2), (65, 6, 2), (130, 2, 1)])
def test_decode_many_sequences(seqs, heads, kv):
    """Ragged batches of 64 sequences and more, idle ones among them; rows of the same as a prefill."""
    r = np.random.default_rng(41)
    lengths = [int(n) for n in np.where(r.random(seqs) < 0.2, 0, np.exp(r.uniform(0, 7, seqs)))]
    pool = Pool(41, "bf16", kv, 64, 16, lengths)
    q = pool.rows(seqs, heads)
    out = pool.cache.decode(q, pool.ints(lengths))
    pool.expect(out, q, range(seqs), [n - 1 for n in lengths])
    out = pool.cache.decode(q, pool.ints(lengths), window=333, sinks=20)
    pool.expect(out, q, range(seqs), [n - 1 for n in lengths], 333, 20)
    if seqs * kv <= 130:
        rows = [[n - 1, n // 2][:int(r.integers(0, 3))] if n else [] for n in lengths]
        _ragged(pool, heads, rows)


@pytest.mark.parametrize("seqs,kv,length", [(64, 8, 30000), (70, 2, 30000), (3, 8, 70000)])
def test_decode_long_sequences_on_the_same_pages(seqs, kv, length):
    """Lengths at which chunks are hundreds of tiles; all tables name the pages of one small pool."""
    from paper_2608_10824_amd.paged import PagedCache
    page, n_pages = 128, 40
    pool = Pool(42, "fp16", kv, 64, page, [page * n_pages], spare=0, extra_columns=0)
    columns = -(-length // page)
    pool.table = pool.r.integers(0, n_pages, (seqs, columns)).astype(np.int32)
    pool.cache = c = PagedCache(pool.cache.k_pages, pool.cache.v_pages, torch.tensor(pool.table, device=DEV))
    lengths = [int(length * f) for f in np.linspace(0.6, 1, seqs)]
    lengths[1] = 5
    q = pool.rows(seqs, kv)
    out = c.decode(q, pool.ints(lengths))
    pick = [0, 1, seqs // 2, seqs - 1]
    pool.expect(out[pick], q[pick], pick, [lengths[i] - 1 for i in pick])


# ------------------------------------- prefill: lists long enough for tiles of 128 rows
def _tiled(pool, rows, heads, window=0, sinks=0):
    """The calls below are of this kind (what sends them there is in k_paged_decode.hip)."""
    slots = pool.table.shape[1] * pool.page
    most = min(window + sinks + 64, slots) if window else slots
    assert rows * heads * most > 1 << 22 and rows * heads // pool.kv > 16 * pool.table.shape[0]


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,dh,page,columns", [(56, 8, 128, 16, 0), (64, 1, 64, 32, 0), (64, 32, 64, 128, 0),
                                                      (53, 1, 128, 64, 0), (6, 2, 128, 16, 195), (5, 1, 64, 128, 26),
                                                      (4, 4, 64, 16, 200)])
def test_tiles_of_ragged_rows(t, heads, kv, dh, page, columns):
    """Whole prompts, one row, no row, chunks behind a cached prefix, rows with
    gaps, rows in falling order; tables that hold the lengths alone, and such
    that the slots are split."""
    pool = Pool(51, t, kv, dh, page, [150, 1, 40, 256, 97, 66], extra_columns=columns)
    rows = [range(150), [0], [], range(197, 256), sorted(pool.r.permutation(97)[:41]), range(65, -1, -1)]
    _tiled(pool, sum(len(x) for x in rows), heads)
    _ragged(pool, heads, rows)


@pytest.mark.parametrize("t,dh,page,kv", [("bf16", 64, 16, 2), ("fp16", 128, 64, 1)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (9, 4), (64, 0), (31, 33), (130, 5), (64, 200), (300, 2)])
def test_tiles_with_window_and_sinks(t, dh, page, kv, window, sinks):
    pool = Pool(52, t, kv, dh, page, [333, 20, 180])
    rows = [range(140, 333), range(20), range(0, 180, 3)]
    heads = ((1 << 22) // (273 * kv * min(window + sinks + 64, 300)) + 1) * kv
    _tiled(pool, 273, heads, window, sinks)
    _ragged(pool, heads, rows, window, sinks)


@pytest.mark.parametrize("t,dh,page", [("bf16", 128, 64), ("fp16", 64, 16), ("bf16", 64, 128), ("fp16", 128, 16)])
def test_tiles_over_many_slots(t, dh, page):
    """Few tiles over thousands of slots, split and joined: in up to sixteen
    parts and in more, with and without a window, and rows that see few of them."""
    pool = Pool(53, t, 1, dh, page, [5100])
    _tiled(pool, 41, 21)
    _ragged(pool, 21, [[5099, 0, 300] + list(range(5062, 5100))])
    _tiled(pool, 90, 30, 1500, 70)
    _ragged(pool, 30, [range(5010, 5100)], 1500, 70)
    pool = Pool(54, t, 2, dh, page, [2000, 130, 900])
    rows = [range(1900, 2000), range(130), [899]]
    _tiled(pool, 231, 10)
    _ragged(pool, 10, rows)


@pytest.mark.parametrize("columns", [0, 200])
def test_tiles_where_rows_see_nothing_or_see_each_other(columns):
    """Empty rows among others and whole tiles of them, an action block whose
    rows give the block's last slot, rows of no sequence before and behind."""
    heads = 80 if columns == 0 else 6
    pool = Pool(55, "bf16", 2, 64, 16, [256, 60], extra_columns=columns)
    lasts = [5] * 7 + [-1, 3, -1, 49] + list(range(90)) + [99] * 30 + [-1] * 90 + [7, -9, 59] + [8] * 6
    n = len(lasts)
    q = pool.rows(n, heads)
    _tiled(pool, n, heads)
    held = torch.full((n, heads, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints([7, n - 9, n - 6]), out=held)
    assert (held[:7] == 5).all() and (held[n - 6:] == 5).all()
    pool.expect(out[7:n - 6], q[7:n - 6], [0] * (n - 16) + [1] * 3, lasts[7:n - 6])


@pytest.mark.parametrize("columns", [0, 200])
def test_tiles_with_pages_that_do_not_exist(columns):
    heads = 72 if columns == 0 else 6
    pool = Pool(56, "fp16", 1, 64, 16, [256, 128, 64], extra_columns=columns)
    c = pool.cache
    for s, col, to in ((0, 0, -1), (0, 3, c.k_pages.shape[0]), (0, 9, -2 ** 31), (1, 2, 2 ** 31 - 1), (2, 0, -7),
                       (2, 1, -1), (2, 2, -1), (2, 3, -1)):
        pool.table[s, col] = to
    c.page_table.copy_(torch.tensor(pool.table))
    _tiled(pool, 250, heads)
    _, out, _, _, _ = _ragged(pool, heads, [range(106, 256), range(40, 128), range(52, 64)])
    assert not out[238:].any()
    # a length over what the table holds ends at the table's last slot
    last = pool.table.shape[1] * 16 - 1
    q = pool.rows(250, heads)
    out = c.prefill(q, pool.ints([2 ** 31 - 1, last + 1] * 125), pool.ints([0, 250, 250, 250]))
    pool.expect(out, q, [0] * 250, [last] * 250)


@pytest.mark.parametrize("t,heads,columns,window,sinks", [("bf16", 72, 0, 0, 0), ("fp16", 72, 0, 0, 0), ("bf16", 6, 180, 0, 0),
                                                          ("fp16", 156, 0, 40, 4), ("bf16", 156, 200, 40, 4)])
@pytest.mark.parametrize("dh", [64, 128])
def test_tiles_keep_nan_and_infinities_with_the_rows_that_see_them(t, heads, columns, window, sinks, dh):
    pool = Pool(57, t, 2, dh, 16, [256], extra_columns=columns)
    c, tb = pool.cache, pool.table
    c.v_pages[tb[0, 5], 0, 3, 7] = float("nan")    # slot 87
    c.v_pages[tb[0, 8], 1, 9, 1] = float("inf")    # slot 129
    c.k_pages[tb[0, 9], 0, 15, 0] = float("nan")   # slot 159
    _tiled(pool, 256, heads, window, sinks)
    _, out, _, _, _ = _ragged(pool, heads, [range(256)], window, sinks)
    o, g = _np(out), heads // 2
    assert np.isfinite(o[:87]).all() and np.isnan(o[87, :g, 3]).all() and np.isfinite(o[:159, g:, :9]).all()
    assert np.isinf(o[129, g:, 9]).all() and np.isnan(o[159, :g]).all()
    if window:
        assert np.isfinite(o[199:]).all()


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_tiles_of_steep_scores(t):
    """The running maximum moves up and down over hundreds."""
    pool = Pool(58, t, 1, 64, 16, [256])
    for j in range(256):
        pool.cache.k_pages[pool.table[0, j // 16], 0, j % 16] *= (j % 50) / 10
    _tiled(pool, 256, 72)
    _ragged(pool, 72, [range(256)], scale=4.0)


def test_tiles_strides_scale_and_out():
    pool = Pool(59, "bf16", 2, 128, 32, [256])
    wide = pool.rows(256, 70)
    q = wide[:, 4:64]
    held = torch.full((256, 62, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    _tiled(pool, 256, 60)
    out = pool.cache.prefill(q, pool.ints(range(256)), pool.ints([0, 256]), scale=0.3, out=held[:, 1:61])
    assert (held[:, 0] == 3).all() and (held[:, 61] == 3).all()
    pool.expect(out, q, [0] * 256, range(256), scale=0.3)


def test_captured_tiles_replay_with_other_rows():
    """A captured call of long lists, split over the slots: rows, bounds and
    the table change between replays; each is bit for bit the eager result."""
    pool = Pool(60, "bf16", 2, 64, 16, [1500, 700], spare=30)
    c = pool.cache
    n, heads = 400, 8
    q, last, begin = pool.rows(n, heads), pool.ints([3] * n), pool.ints([0, 200, n])
    _tiled(pool, n, heads)
    graphs, outs = [], []
    c.prefill(q, last, begin)
    torch.cuda.synchronize()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.prefill(q, last, begin))
        graphs.append(g)
    for turn, (cut, a, b) in enumerate([(200, 1499, 699), (350, 1499, 60), (10, 20, 699), (400, 1100, -1)]):
        q.copy_(pool.rows(n, heads))
        lasts = [max(a - cut + 1 + i, -1) for i in range(cut)] + [max(b - n + cut + 1 + i, -1) for i in range(n - cut)]
        last.copy_(pool.ints(lasts))
        begin.copy_(pool.ints([0, cut, n]))
        want = c.prefill(q, last, begin)
        if turn < 2:
            pick = list(range(0, n, 23)) + [cut - 1, n - 1]
            pool.expect(want[pick], q[pick], [int(i >= cut) for i in pick], [lasts[i] for i in pick])
        for g, got in zip(graphs, outs):
            got.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(want, got)


# ------------------------------------------------------- workspaces of split calls
def test_a_workspace_may_hold_anything():
    """Split decodes and prefills through the C ABI, in memory that holds zeros,
    ones, noise, another call's rest and their own: the same bits."""
    from paper_2608_10824_amd import gvc
    pool = Pool(61, "bf16", 2, 128, 16, [4000, 17, 2100, 0])
    c = pool.cache
    desc = gvc.PagedDesc(gvc.BF16, 8, 2, 128, 16, c.k_pages.shape[0], 4, c.page_table.shape[1])
    q, lengths, begin = pool.rows(20, 8), pool.ints([4000, 17, 2100, 0]), pool.ints([0, 1, 2, 20, 20])
    last = pool.ints([3999, 16] + list(range(2082, 2100)))
    long_q, long_last, long_begin = pool.rows(300, 8), pool.ints(range(1800, 2100)), pool.ints([0, 0, 0, 300, 300])
    pages = (c.k_pages.data_ptr(), c.v_pages.data_ptr(), c.page_table.data_ptr())
    sizes = [gvc.paged_workspace(desc, False, 4), gvc.paged_workspace(desc, True, 20), gvc.paged_workspace(desc, True, 300)]
    assert min(sizes) > 0
    work = torch.zeros(max(sizes), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream

    def run():
        outs = [torch.empty_like(x) for x in (q[:4], q, long_q)]
        gvc.paged_decode(desc, 0.09, 0, 0, q.data_ptr(), 1024, lengths.data_ptr(), *pages, outs[0].data_ptr(), 1024,
                         work.data_ptr(), sizes[0], stream)
        gvc.paged_prefill(desc, 0.09, 0, 0, q.data_ptr(), 1024, last.data_ptr(), begin.data_ptr(), 20, *pages,
                          outs[1].data_ptr(), 1024, work.data_ptr(), sizes[1], stream)
        gvc.paged_prefill(desc, 0.09, 0, 0, long_q.data_ptr(), 1024, long_last.data_ptr(), long_begin.data_ptr(), 300,
                          *pages, outs[2].data_ptr(), 1024, work.data_ptr(), sizes[2], stream)
        return outs

    want = run()
    pool.expect(want[0], q[:4], range(4), [3999, 16, 2099, -1], scale=0.09)
    pool.expect(want[1], q, [0, 1] + [2] * 18, [3999, 16] + list(range(2082, 2100)), scale=0.09)
    noise = torch.randint(0, 256, work.shape, dtype=torch.uint8, device=DEV)
    for fill in (None, 255, 1, noise):
        if fill is not None:
            work.copy_(noise) if fill is noise else work.fill_(fill)
        for x, y in zip(want, run()):
            assert torch.equal(x, y)


def test_a_captured_split_call_after_bounds_that_fall():
    """What a replay with wrong bounds leaves in the workspace does not reach
    the next one (few rows, whose parts count each other; bounds that fall can
    name more parts than the call has)."""
    from paper_2608_10824_amd.paged import PagedCache
    pool = Pool(62, "bf16", 1, 64, 16, [2000])
    n, seqs = 30, 40
    pool.table = np.repeat(pool.table, seqs, 0)
    pool.cache = c = PagedCache(pool.cache.k_pages, pool.cache.v_pages, torch.tensor(pool.table, device=DEV))
    q, last = pool.rows(n, 16), pool.ints([1999] * n)
    right = [0, 10, 20] + [n] * (seqs - 2)
    begin = pool.ints(right)
    assert n * 16 * 2032 < 1 << 21
    want = c.prefill(q, last, begin)
    pool.expect(want[::9], q[::9], [0, 0, 1, 2], [1999] * 4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = c.prefill(q, last, begin)
    for wrong in ([0, n] * (seqs // 2) + [0], [n, 0] * (seqs // 2) + [n], [0, n, 1, n] * (seqs // 4) + [n]):
        begin.copy_(pool.ints(wrong))
        g.replay()
        torch.cuda.synchronize()
        begin.copy_(pool.ints(right))
        got.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, got)


# ----------------------------------------------------------------- together
def test_a_history_appended_and_attended():
    """Two sequences from an empty cache: a prompt, a second chunk, then single
    tokens; each step's attention over what has been appended so far."""
    from paper_2608_10824_amd.paged import PagedCache
    heads, kv, dh, page = 6, 2, 128, 16
    c = PagedCache.empty(30, page, kv, dh, 2, 12, device=DEV)
    assert (c.page_table == -1).all()
    ids = np.random.default_rng(31).permutation(30)[:24].reshape(2, 12)
    c.page_table.copy_(torch.tensor(ids.astype(np.int32)))
    pool = Pool.__new__(Pool)
    pool.r, pool.t, pool.dh, pool.cache, pool.table = np.random.default_rng(32), "bf16", dh, c, ids
    have = [0, 0]
    gain = torch.ones(dh, dtype=torch.bfloat16, device=DEV)
    for step, new in enumerate([(40, 25), (30, 61), (1, 1), (1, 0), (1, 1)]):
        rows = [(s, have[s] + i) for s in range(2) for i in range(new[s])]
        n = len(rows)
        seq, slot = pool.ints([s for s, _ in rows]), pool.ints([j for _, j in rows])
        pos = pool.ints([[j // 9 + 5, j % 9 // 3, j % 3] for _, j in rows]).T.contiguous()
        x = pool.rows(n, heads + 2 * kv)
        c.check(pool.ints([have[s] + new[s] for s in range(2)]), seq, slot)
        q = c.append(x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], seq, slot, positions=pos,
                     rope_pairs=(16, 24, 24), q_norm=gain, k_norm=gain)
        for i, (s, j) in enumerate(rows):   # the values arrived
            assert torch.equal(c.v_pages[ids[s, j // page], :, :, j % page], x[i, heads + kv:])
        have = [have[s] + new[s] for s in range(2)]
        if max(new) > 1:
            begin = [0, new[0], new[0] + new[1]]
            out = c.prefill(q, slot, pool.ints(begin), window=50, sinks=4)
            pool.expect(out, q, [s for s, _ in rows], [j for _, j in rows], 50, 4)
        elif min(new) == 1:
            out = c.decode(q, pool.ints(have), window=50, sinks=4)
            pool.expect(out, q, [0, 1], [have[0] - 1, have[1] - 1], 50, 4)


def test_captured_calls_replay_beside_eager_ones():
    """One graph of append, decode and prefill, replayed with new inputs and a
    changed table, eager calls and a second graph's replays between: each
    replay is bit for bit the eager result."""
    pool = Pool(33, "bf16", 2, 64, 16, [90, 700, 1], spare=60)
    c = pool.cache
    q, k, v = pool.rows(3, 8), pool.rows(3, 2), pool.rows(3, 2)
    seq, slot, lengths = pool.ints([0, 1, 2]), pool.ints([89, 699, 0]), pool.ints([90, 700, 1])
    last, begin = pool.ints([89, 699, 0]), pool.ints([0, 1, 2, 3])

    def step():
        r = c.append(q, k, v, seq, slot)
        return r, c.decode(r, lengths), c.prefill(r, last, begin, window=64, sinks=3)

    step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    spare = [i for i in range(c.k_pages.shape[0]) if i not in set(pool.table.flatten())]
    for turn in range(4):
        q.copy_(pool.rows(3, 8))
        k.copy_(pool.rows(3, 2))
        slot.copy_(pool.ints([89, 699 - turn, 0]))
        lengths.copy_(pool.ints([90 - turn, 700, turn % 2]))
        if turn == 2:   # the second sequence's first page moves
            c.k_pages[spare[0]], c.v_pages[spare[0]] = c.k_pages[pool.table[1, 0]], c.v_pages[pool.table[1, 0]]
            c.page_table[1, 0] = spare[0]
        want = step()
        for g, got in zip(graphs, outs):
            for x in got:
                x.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(want, got):
                assert torch.equal(x, y)


def test_two_streams_at_once():
    pool = Pool(34, "bf16", 2, 128, 16, [1500, 40])
    c = pool.cache
    lengths = pool.ints([1500, 40])
    qs = [pool.rows(2, 8) for _ in range(6)]
    want = [c.decode(q, lengths) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i, q in enumerate(qs):
        with torch.cuda.stream(streams[i % 2]):
            got.append(c.decode(q, lengths))
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x, y)


def test_pool_over_four_gib():
    """Pages whose byte offsets pass 32 bits (and element offsets 31)."""
    from paper_2608_10824_amd.paged import PagedCache
    kv, dh, page, n_pages = 8, 128, 128, 17500   # 4.3 GiB each of keys and values
    c = PagedCache.empty(n_pages, page, kv, dh, 2, 4, device=DEV)
    pages = np.array([[n_pages - 1, 3, n_pages - 2, 8200], [1, n_pages - 3, 2, 0]], dtype=np.int32)
    c.page_table.copy_(torch.tensor(pages))
    g = torch.Generator(device=DEV).manual_seed(35)
    n = 400
    x = torch.randn(n, 32, dh, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = x[:, :16], x[:, 16:24], x[:, 24:]
    seq = torch.tensor([i % 2 for i in range(n)], dtype=torch.int32, device=DEV)
    slot = torch.tensor([i // 2 for i in range(n)], dtype=torch.int32, device=DEV) + 200
    r = c.append(q, k, v, seq, slot, rope_pairs=())
    assert torch.equal(r, q)
    for s, j, i in ((0, 399, 398), (0, 256, 112), (1, 255, 111), (1, 200, 1)):
        assert torch.equal(c.k_pages[pages[s, j // page], :, j % page], k[i])
        assert torch.equal(c.v_pages[pages[s, j // page], :, :, j % page], v[i])
    # a small pool with the same pages gives the same attention
    small = PagedCache(c.k_pages[pages.flatten()].clone(), c.v_pages[pages.flatten()].clone(),
                       torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4))
    qd = q[:2].contiguous()
    lengths = torch.tensor([400, 399], dtype=torch.int32, device=DEV)
    assert torch.equal(c.decode(qd, lengths), small.decode(qd, lengths))
    last = torch.tensor([399, 120, 399], dtype=torch.int32, device=DEV)
    begin = torch.tensor([0, 2, 3], dtype=torch.int32, device=DEV)
    qp = q[:3].contiguous()
    assert torch.equal(c.prefill(qp, last, begin), small.prefill(qp, last, begin))


def test_outputs_in_place_of_their_inputs():
    """q_out or out may be q itself: rotation, unsplit and split decodes and
    lists of rows of both kinds give the same bits."""
    pool = Pool(37, "bf16", 2, 64, 16, [1500, 40, 0], extra_columns=20)
    c, n = pool.cache, 300
    x = pool.rows(n, 12)
    seq, slot = pool.ints([0] * n), pool.ints(range(1200, 1500))
    want = c.append(x[:, :8], x[:, 8:10], x[:, 10:], seq, slot)
    got = x.clone()
    c.append(got[:, :8], got[:, 8:10], got[:, 10:], seq, slot, q_out=got[:, :8])
    assert torch.equal(want, got[:, :8]) and torch.equal(x[:, 8:], got[:, 8:])
    for f in (lambda q, o: c.decode(q, pool.ints([1500, 40, 0]), out=o), lambda q, o: c.decode(q, pool.ints([300, 40, 0]), out=o),
              lambda q, o: c.prefill(q, pool.ints([1499, 39, 7]), pool.ints([0, 1, 3, 3]), out=o)):
        q = pool.rows(3, 8)
        want = f(q, None)
        assert torch.equal(f(q, q), want)
    q = pool.rows(n, 8)
    _tiled(pool, n, 8)
    want = c.prefill(q, slot, pool.ints([0, n, n, n]))
    assert torch.equal(c.prefill(q, slot, pool.ints([0, n, n, n]), out=q), want)
    pool = Pool(38, "fp16", 1, 128, 32, [256], extra_columns=0)
    q, slot = pool.rows(256, 72), pool.ints(range(256))
    _tiled(pool, 256, 72)
    want = pool.cache.prefill(q, slot, pool.ints([0, 256]))
    assert torch.equal(pool.cache.prefill(q, slot, pool.ints([0, 256]), out=q), want)


def test_more_wrapper_refusals():
    from paper_2608_10824_amd.paged import PagedCache
    pool = Pool(39, "bf16", 2, 64, 16, [20, 20])
    c, q, two = pool.cache, pool.rows(2, 4), pool.ints([3, 4])
    for f in (lambda: c.decode(q, two, window=2 ** 32 + 5), lambda: c.decode(q, two, sinks=2 ** 31),
              lambda: c.prefill(q, two, pool.ints([0, 1, 2]), window=2 ** 31),
              lambda: PagedCache(c.k_pages.clone().requires_grad_(), c.v_pages, c.page_table)):
        with pytest.raises(ValueError):
            f()


def test_wrapper_refusals():
    pool = Pool(36, "bf16", 2, 64, 16, [20, 20])
    c = pool.cache
    q, k, v, two = pool.rows(2, 4), pool.rows(2, 2), pool.rows(2, 2), pool.ints([3, 4])
    bad = [lambda: c.decode(q.half(), two), lambda: c.decode(q[:1], two), lambda: c.decode(q, two.long()),
           lambda: c.decode(q, two[:1]), lambda: c.decode(q.cpu(), two), lambda: c.decode(q[..., :32], two),
           lambda: c.decode(q.transpose(1, 2), two), lambda: c.decode(q, two, out=q[:, :2]),
           lambda: c.decode(q[0], two), lambda: c.decode(q.clone().requires_grad_(), two),
           lambda: c.prefill(q, two, two), lambda: c.prefill(q, two[:1], pool.ints([0, 1, 2])),
           lambda: c.append(q, k, v[:1], two, two), lambda: c.append(q, k[:, :1], v, two, two),
           lambda: c.append(q, k, v, two, two[:1]), lambda: c.append(q, k, v, two, two, rope_pairs=(8, 8, 8, 8)),
           lambda: c.append(q, k, v, two, two, positions=two), lambda: c.append(None, k, v, two, two, q_out=q),
           lambda: c.append(q, k, v, two, two, q_norm=q[0, 0, :32]), lambda: c.append(q[:1], k, v, two, two)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    from paper_2608_10824_amd import gvc
    for f in (lambda: c.decode(q, two, scale=0.0), lambda: c.decode(q, two, window=-1), lambda: c.prefill(q[:, :3], two, pool.ints([0, 1, 2])),
              lambda: c.append(q, k, v, two, two, rope_pairs=(33,)), lambda: c.append(q, k, v, two, two, rms_eps=-1.0)):
        with pytest.raises(gvc.GvcError):
            f()


# ------------------------------------------- values near the end of the type's range
def _large(pool, power):
    """The pool's values up to 2^(power + 2), all of one sign: their sums before the division are larger."""
    pool.cache.v_pages.abs_().clamp_(max=4).mul_(2.0 ** power)


@pytest.mark.parametrize("power", [90, 114, 121, 125])
def test_outputs_are_finite_where_sums_overflow(power):
    """bf16 values to 2^127: decode (split and not, with a window) and lists of few rows give
    the finite outputs of their formulas."""
    lengths = [1, 40, 700, 3000, 0]
    pool = Pool(63, "bf16", 2, 64, 16, lengths)
    _large(pool, power)
    q = pool.rows(5, 8, 2.0)
    pool.expect(pool.cache.decode(q, pool.ints(lengths)), q, range(5), [n - 1 for n in lengths])
    pool.expect(pool.cache.decode(q, pool.ints(lengths), window=300, sinks=20), q, range(5), [n - 1 for n in lengths], 300, 20)
    _ragged(pool, 8, [[0], range(40), [699, 3], [2999], []])
    pool = Pool(64, "bf16", 1, 128, 32, [300, 33], extra_columns=0)
    _large(pool, power)
    q = pool.rows(2, 20, 2.0)
    pool.expect(pool.cache.decode(q, pool.ints([300, 33])), q, range(2), [299, 32])


@pytest.mark.parametrize("power", [90, 114, 121, 125])
@pytest.mark.parametrize("dh,heads,columns", [(64, 72, 0), (128, 72, 0), (64, 6, 200), (128, 6, 200)])
def test_tiles_are_finite_where_sums_overflow(power, dh, heads, columns):
    pool = Pool(65, "bf16", 2, dh, 16, [256], extra_columns=columns)
    _large(pool, power)
    _tiled(pool, 256, heads)
    _ragged(pool, heads, [range(256)])


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("form", ["decode", "split decode", "rows", "split rows", "tiles", "split tiles"])
def test_rounded_probabilities_do_not_carry_an_output_past_the_largest_value(t, form):
    """Every value is the type's largest, so every output is.  One slot of 32 has the most weight, the others just over
    half of it, which 16 bits round up by almost u: more than from the largest value half way to the next."""
    n = 2000 if form.startswith("split") else 350
    tiles = form.endswith("tiles")
    pool = Pool(66, t, 1, 64, 16, [n], extra_columns=1)
    c, big, rows = pool.cache, torch.finfo(TYPES[t]).max, 300 if tiles else 1
    c.v_pages.copy_(torch.where(c.v_pages.isnan(), c.v_pages, torch.full_like(c.v_pages, big)))
    c.k_pages.copy_(torch.where(c.k_pages.isnan(), c.k_pages, torch.zeros_like(c.k_pages)))
    for j in range(n):
        c.k_pages[pool.table[0, j // 16], 0, j % 16, 0] = -1.0 if j % 32 else 0.0
    scale = -np.log((1 + 1.1 * _u(t)) / 2)
    heads = 2 if not tiles else 42 if n < 1000 else 8
    q = torch.zeros(rows, heads, 64, dtype=TYPES[t], device=DEV)
    q[:, :, 0] = 1
    if tiles:
        _tiled(pool, rows, heads)
    if form.endswith("decode"):
        out = c.decode(q, pool.ints([n]), scale=scale)
    else:
        out = c.prefill(q, pool.ints([n - 1] * rows), pool.ints([0, rows]), scale=scale)
    assert (out == big).all()
    out = c.prefill(-q, pool.ints([n - 1] * rows), pool.ints([0, rows]), scale=scale)
    assert (out == big).all()
    c.v_pages[pool.table[0, 0], 0, 7, 3] = float("-inf")   # an infinity in sight stays one
    out = c.prefill(q, pool.ints([n - 1] * rows), pool.ints([0, rows]), scale=scale)
    assert (out[:, :, 7] == float("-inf")).all() and (out[:, :, :7] == big).all() and (out[:, :, 8:] == big).all()


def test_gains_that_are_parameters():
    pool = Pool(68, "bf16", 2, 64, 16, [20, 20])
    c, seq, slot = pool.cache, pool.ints([0, 1]), pool.ints([3, 4])
    q, k, v = pool.rows(2, 4), pool.rows(2, 2), pool.rows(2, 2)
    gain = torch.tensor(1 + 0.2 * pool.r.standard_normal(64)).to(torch.bfloat16).to(DEV)
    want = c.append(q, k, v, seq, slot, q_norm=gain, k_norm=gain)
    param = torch.nn.Parameter(gain.clone())
    with torch.no_grad():
        got = c.append(torch.nn.Parameter(q), k, v, seq, slot, q_norm=param, k_norm=param)
    assert torch.equal(want, got) and not got.requires_grad
    with pytest.raises(ValueError):
        c.append(q, k, v, seq, slot, q_norm=param)


# ------------------------- calls of many sequences, many heads and large pools, by the path that they take
def _fused(pool, window=0, sinks=0):
    """(tiles of slots that a row sees at most, chunk length, whether units join themselves) as in k_paged_decode.hip."""
    slots = pool.table.shape[1] * pool.page
    most = min(-(-window // 32) + 1 + -(-sinks // 32) if window else 2 ** 30, -(-slots // 32))
    least = -(-most // 8)
    return most, least, least <= 8 or (least <= 32 and pool.kv * 8 >= 256)


@pytest.mark.parametrize("t,dh,heads,kv", [("bf16", 64, 32, 32), ("fp16", 64, 64, 32), ("bf16", 128, 34, 34)])
def test_units_of_many_heads_join_long_chunks_themselves(t, dh, heads, kv):
    """2100 to 8192 slots of at least 32 key-value heads: eight long chunks and no second launch."""
    lengths = [2700, 300, 0, 2100]
    pool = Pool(71, t, kv, dh, 16, lengths, extra_columns=300)
    most, least, fused = _fused(pool)
    assert 64 < most <= 256 and least > 8 and fused
    q = pool.rows(4, heads, 2.0)
    for _ in range(2):   # the second in memory that the first has left
        pool.expect(pool.cache.decode(q, pool.ints(lengths)), q, range(4), [n - 1 for n in lengths])
    assert _fused(pool, 2200, 40)[1:] == (9, True)
    pool.expect(pool.cache.decode(q, pool.ints(lengths), window=2200, sinks=40), q, range(4), [n - 1 for n in lengths], 2200, 40)
    if 4 * kv <= 128:
        rows = [range(2690, 2700), [299, 0], [], [2099]]
        assert sum(len(x) for x in rows) * heads // kv <= 4 * 16
        _ragged(pool, heads, rows)


@pytest.mark.parametrize("seqs,kv,heads,columns", [(65, 2, 40, 0), (130, 2, 40, 0), (70, 1, 12, 200)])
def test_tiles_of_many_sequences(seqs, kv, heads, columns):
    """More sequences than a wave has lanes, some without rows, rows of no sequence before and behind."""
    r = np.random.default_rng(72)
    lengths = [int(n) for n in r.integers(0, 90, seqs)]
    lengths[0], lengths[seqs - 1] = 90, 33
    pool = Pool(72, "bf16", kv, 64, 16, lengths, extra_columns=columns)
    lasts, seq, begin = [5] * 3, [-1] * 3, [3]
    for s, n in enumerate(lengths):
        new = 0 if s % 7 == 3 else min(n, int(r.integers(0, 60)))
        lasts += range(n - new, n)
        seq += [s] * new
        begin.append(len(lasts))
    lasts, seq = lasts + [4] * 5, seq + [-1] * 5
    n = len(lasts)
    _tiled(pool, n, heads)
    q = pool.rows(n, heads, 2.0)
    held = torch.full((n, heads, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints(begin), out=held)
    assert (held[:3] == 5).all() and (held[n - 5:] == 5).all()
    pick = sorted({x for s in range(seqs) for x in (begin[s], begin[s + 1] - 1) if begin[s + 1] > begin[s]})
    assert seq[pick[-1]] > 64 or seqs == 65
    pool.expect(out[pick], q[pick], [seq[i] for i in pick], [lasts[i] for i in pick])


@pytest.mark.parametrize("seqs,kv,columns", [(70, 2, 1000), (40, 4, 1700)])
def test_tiles_of_one_row_to_a_sequence(seqs, kv, columns):
    """One row of each of many sequences over a large table: 128-row tiles, whole and split over the slots."""
    r = np.random.default_rng(73)
    lengths = [int(n) for n in np.exp(r.uniform(0, 7, seqs))]
    lengths[-1] = 1900
    pool = Pool(73, "fp16", kv, 64, 16, lengths, extra_columns=columns)
    heads = 2 * kv
    assert seqs * heads * pool.table.shape[1] * 16 > 1 << 22 and seqs * kv > 128
    _ragged(pool, heads, [[n - 1] for n in lengths])


@pytest.mark.parametrize("length,fused", [(1500, True), (3000, False)])
def test_few_rows_of_many_sequences(length, fused):
    """Lists of few rows in 70 sequences, joined by their units and by a second launch, which looks a row's sequence up."""
    r = np.random.default_rng(74)
    lengths = [int(n) for n in r.integers(1, 100, 70)]
    lengths[3], lengths[66] = length, length - 400
    pool = Pool(74, "bf16", 1, 64, 16, lengths)
    assert _fused(pool)[2] == fused
    rows = [[n - 1] if s % 3 else [] for s, n in enumerate(lengths)]
    rows[3], rows[66], rows[69] = [length - 1, 7], [length - 401, length - 402, 900], [0]
    assert sum(len(x) for x in rows) * 8 <= 70 * 16
    _ragged(pool, 8, rows)


def test_tiles_over_four_gib():
    """Pages whose byte offsets pass 32 bits, and a list long enough for 128-row tiles: the same bits as from a small pool."""
    from paper_2608_10824_amd.paged import PagedCache
    kv, dh, page, n_pages = 8, 128, 128, 17500   # 4.3 GiB each of keys and values
    c = PagedCache.empty(n_pages, page, kv, dh, 2, 4, device=DEV)
    pages = np.array([[n_pages - 1, 3, n_pages - 2, 8200], [1, n_pages - 3, 2, 0]], dtype=np.int32)
    c.page_table.copy_(torch.tensor(pages))
    g = torch.Generator(device=DEV).manual_seed(75)
    for i in pages.flatten().tolist():
        c.k_pages[i] = torch.randn(kv, page, dh, generator=g, device=DEV)
        c.v_pages[i] = torch.randn(kv, dh, page, generator=g, device=DEV)
    pool = Pool.__new__(Pool)
    pool.t, pool.kv, pool.dh, pool.page, pool.table = "bf16", kv, dh, page, np.arange(8).reshape(2, 4)
    at = torch.tensor(pages.flatten().astype(np.int64), device=DEV)
    pool.cache = PagedCache(c.k_pages[at].clone(), c.v_pages[at].clone(), torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4))
    lasts = list(range(512)) + list(range(400, 500))
    n = len(lasts)
    q = torch.randn(n, 16, dh, generator=g, device=DEV).to(torch.bfloat16)
    _tiled(pool, n, 16)
    args = (q, torch.tensor(lasts, dtype=torch.int32, device=DEV), torch.tensor([0, 512, n], dtype=torch.int32, device=DEV))
    out = c.prefill(*args)
    assert torch.equal(out, pool.cache.prefill(*args))
    pick = [0, 130, 511, 512, n - 1]
    pool.expect(out[pick], q[pick], [0, 0, 0, 1, 1], [lasts[i] for i in pick])
