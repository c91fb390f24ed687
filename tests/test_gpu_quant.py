"""The quantised paged cache's operators against their float64 oracle, through
QuantPagedCache (and so through the C ABI).

Bounds (none is fitted).  Attention is held to oracle/paged.py over what the
codes stand for (rounded once to the 16-bit type), within the bounds that
tests/test_gpu_paged.py derives for the 16-bit cache: scores, exponentials
and sums in fp32, each probability rounded once to 16 bits, the output once.
 Values are quantised as they come: codes and scales have to be the oracle's, bit
for bit.  Keys are computed in double: below position 2^17 an angle is off by at most 2^17 turns times 64
roundings, 2^-30, and mostly by 2^-36, so that a value in 2^26 could be half way between two codes within that: codes
and scales have to be the oracle's, bit for bit.  (A seed that hit one would fail once and always; none does.)  At
farther positions a key is off by d, what tests/test_gpu_paged.py allows
before the rounding: its scale has to be that of a head whose largest magnitude
is within d of the exact one's, and what a code stands for is within half
a step of it (2^-4 of the value, 2^-10 of the scale below 2^-6 of it) and d of the exact key.
 Reading back computes nothing but one rounding: bit for bit.
"""
import numpy as np
import pytest
import torch

from oracle import paged as op
from oracle import quant as oq
from tests import test_gpu_paged as paged
from tests.test_gpu_paged import DEV, TYPES, _np, _ragged, _tiled, _tiny, _u

pytestmark = pytest.mark.gpu


class Values:
    """A quantised cache's keys and values as float64 arrays, in the places of a 16-bit cache's tensors."""

    def __init__(self, c, t):
        b = [x.view(torch.uint8).cpu().numpy() for x in (c.k_pages, c.k_scales, c.v_pages, c.v_scales)]
        self.k_pages = torch.tensor(oq.values(b[0], b[1], t))
        self.v_pages = torch.tensor(oq.values(b[2].swapaxes(2, 3), b[3], t).swapaxes(2, 3))


class Pool(paged.Pool):
    """As in the tests of the 16-bit cache, quantised: heads of sizes 2^-3 to 2^3; codes and scales that no
    sequence holds are NaN."""

    def __init__(self, seed, t, kv, dh, page, lengths, spare=2, extra_columns=2):
        super().__init__(seed, t, kv, dh, page, lengths, spare, extra_columns)
        c = self.cache
        n = c.k_pages.shape[0]
        size = 2.0 ** self.r.integers(-3, 4, (2, n, kv, page, 1))
        k, v = _np(c.k_pages) * size[0] / 2, _np(c.v_pages).swapaxes(2, 3) * size[1]
        (kc, ks), (vc, vs) = oq.quantise_heads(k, t), oq.quantise_heads(v, t)
        nobody = np.isnan(k).all(-1)
        ks[nobody] = vs[nobody] = 255
        self.cache = self.of(kc, ks, vc, vs, self.table, t)

    @staticmethod
    def of(k, ks, v, vs, table, t):
        """A cache of codes [pages][kv][page][dh] (v too) and scale codes."""
        from paper_2608_10824_amd.paged import QuantPagedCache
        tensors = [torch.tensor(np.ascontiguousarray(x), device=DEV) for x in (k, ks, v.swapaxes(2, 3), vs)]
        views = (torch.float8_e4m3fn, torch.float8_e8m0fnu) * 2
        return QuantPagedCache(*(x.view(w) for x, w in zip(tensors, views)), torch.tensor(table, device=DEV), TYPES[t])

    def bytes(self):
        """Views of the codes and scales as they are stored: k, k scales, v, v scales."""
        c = self.cache
        return [x.view(torch.uint8) for x in (c.k_pages, c.k_scales, c.v_pages, c.v_scales)]

    def expect(self, out, q, seqs, lasts, window=0, sinks=0, scale=None, least=0.0):
        """Compares attention outputs with the oracle's, row by row (the bounds of the 16-bit cache's tests,
        and `least` more)."""
        val = Values(self.cache, self.t)
        k, v, q, out = val.k_pages.numpy(), val.v_pages.numpy(), _np(q), _np(out)
        scale = self.dh ** -0.5 if scale is None else scale
        u, vmax = _u(self.t), np.abs(v[np.isfinite(v)]).max(initial=0)
        for r, (s, last) in enumerate(zip(seqs, lasts)):
            want, mag, top, n = op.attend_row(q[r], s, last, k, v, self.table, scale, window, sinks)
            if n == 0:
                assert not out[r].any(), "row %d sees nothing and is not zero" % r
                continue
            assert np.array_equal(np.isnan(out[r]), np.isnan(want)), "row %d: NaN" % r
            fine, inf = np.isfinite(want), np.isinf(want)
            assert np.array_equal(out[r][inf], want[inf]), "row %d: inf" % r
            p = (2 * (self.dh + 8) * 2.0 ** -23 * top + (n + 64) * 2.0 ** -23 + u)[:, None]
            with np.errstate(invalid="ignore"):
                tol = u * np.abs(want) + mag * p * (1 + u) + _tiny(self.t) * (1 + n / 64 * vmax) + least
                over = (np.abs(out[r] - want) - tol)[fine]
            assert over.max(initial=0) <= 0, "row %d (sequence %d, last %d): %.3g over its bound" % (r, s, last, over.max())


# ------------------------------------------------------------------- append
def _append(seed, t, heads, kv, dh, page, lengths, rows, pairs=None, positions=None, norm=False, fused=True,
            theta=1e4, eps=1e-5, with_q=True, q_out=None, change=None):
    """Appends rows (sequence, slot) and checks q_out and the whole pool."""
    pool = Pool(seed, t, kv, dh, page, lengths)
    n, r = len(rows), pool.r
    if fused:
        x = pool.rows(n, heads + 2 * kv)
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    else:
        q, k, v = pool.rows(n, heads), pool.rows(n, kv), pool.rows(n, kv)
    if change:
        change(q, k, v)
    gains = [torch.tensor(1 + 0.2 * r.standard_normal(dh)).to(TYPES[t]).to(DEV) if norm else None for _ in range(2)]
    c = pool.cache
    held = [x.clone() for x in pool.bytes()]
    pos = None if positions is None else pool.ints(positions).reshape(-1, n)
    got = c.append(q if with_q else None, k, v, pool.ints([s for s, _ in rows]), pool.ints([j for _, j in rows]),
                   positions=pos, rope_pairs=pairs, rope_theta=theta, q_norm=gains[0], k_norm=gains[1], rms_eps=eps,
                   q_out=q_out)
    want_pairs = (dh // 2,) if pairs is None else pairs

    def exact(x, row, gain):
        """The rotated heads x [heads][dh] of a row, and d."""
        p = [rows[row][1]] * 3 if positions is None else [positions[a][row] for a in range(len(want_pairs))]
        want, mag = np.empty_like(x), np.empty_like(x)
        for h in range(x.shape[0]):
            normed = x[h] / np.sqrt(np.mean(x[h] ** 2) + eps) * gain if gain is not None else x[h]
            want[h] = op.rope_norm(x[h], p, want_pairs, theta, gain, eps)
            m = sum(want_pairs)
            mag[h] = np.abs(normed)
            mag[h, :2 * m] = np.tile(mag[h, :m] + mag[h, m:2 * m], 2)
        return want, mag * (2.0 ** -20 + (dh + 8) * 2.0 ** -24)

    qn, kn, vn = _np(q), _np(k), _np(v)
    gq, gk = [None if g is None else _np(g) for g in gains]
    if with_q:
        assert got.shape == q.shape
        o = _np(got)
        for i in range(n):
            want, d = exact(qn[i], i, gq)
            with np.errstate(invalid="ignore"):
                ok = np.abs(o[i] - want) <= _u(t) * np.abs(want) + d * (1 + _u(t)) + _tiny(t)
            assert (ok | ~np.isfinite(want)).all(), "query %d" % i
    else:
        assert got is None
    ko, kso, vo, vso = [x.cpu().numpy() for x in pool.bytes()]
    near = max(abs(int(x)) for p in ([[j for _, j in rows]] if positions is None else positions) for x in p) < 2 ** 17
    for i, (s, j) in enumerate(rows):
        at = op.place(pool.table, c.k_pages.shape[0], page, s, j)
        if at is None:
            continue
        p, off = at
        want, d = exact(kn[i], i, gk)
        codes, scales = oq.quantise_heads(vn[i], t)
        assert np.array_equal(vso[p, :, off], scales), "scale of value %d" % i
        nan = (codes & 127) == 127
        assert np.array_equal(vo[p, :, :, off][~nan], codes[~nan]) and ((vo[p, :, :, off][nan] & 127) == 127).all(), i
        for h in range(kv):
            fine = np.isfinite(want[h])
            assert np.array_equal((ko[p, h, off] & 127) == 127, ~fine), "key %d: NaN" % i
            if near:
                codes, code = oq.quantise(want[h], t)
                assert kso[p, h, off] == code and np.array_equal(ko[p, h, off][fine], codes[fine]), "key %d" % i
                continue
            w, dd = oq.bounded(want[h], t), np.where(fine, d[h], 0)
            most = np.abs(w[fine]).max(initial=0)
            low, high = (oq.scale_code(np.array([max(most + x, 0)])) for x in (-dd.max(), dd.max()))
            assert low <= kso[p, h, off] <= high, "scale of key %d" % i
            scale = 2.0 ** (float(kso[p, h, off]) - 127)
            step = np.maximum(2.0 ** -4 * (np.abs(w) + dd), 2.0 ** -10 * scale)
            off_by = np.abs(oq.E4M3[ko[p, h, off]] * scale - w)
            assert (off_by <= step + dd)[fine].all(), "key %d: %.3g of the bound" % (i, (off_by / (step + dd))[fine].max())
        # put the slot back: what remains has to be as it was, bit for bit
        for x, y, at in zip(pool.bytes(), held, ((p, slice(None), off),) * 2 + ((p, slice(None), slice(None), off), (p, slice(None), off))):
            x[at] = y[at]
    for x, y in zip(pool.bytes(), held):
        assert torch.equal(x, y)
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


@pytest.mark.parametrize("theta", [1e6, 10000 * 8 ** (128 / 126), 0.7])
def test_append_far_positions(theta):
    far = [0, 1, 10 ** 5, 10 ** 6 + 1, 10 ** 7 + 3, 123456789, 2 ** 31 - 1, -1, -2 ** 31]
    _append(3, "fp16", 2, 2, 128, 16, [9], [(0, j) for j in range(9)], positions=[far], pairs=(64,), theta=theta)


def test_append_rows_in_any_order_of_any_run_length():
    r = np.random.default_rng(4)
    every = [(s, j) for s, n in enumerate([50, 33, 0, 129]) for j in range(n)]
    for n in (1, 2, 15, 63, 64, 65, 150):
        _append(5 + n, "bf16", 4, 2, 64, 16, [50, 33, 0, 129], [every[i] for i in r.permutation(len(every))[:n]])


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("first", range(0, 17, 3))
def test_append_runs_at_any_offset(first, page):
    _append(40 + first, "fp16", 2, 2, 128, page, [400], [(0, first + j) for j in range(300)], fused=False)


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


def test_a_long_append_is_its_parts():
    """A call that passes more than the last cache holds, in one and in three: the same bits everywhere."""
    from paper_2608_10824_amd.paged import QuantPagedCache
    heads, kv, dh, page, n = 32, 8, 128, 32, 13001
    assert n * (4 * heads + 6 * kv) * dh > 256 << 20 and n // 3 * (4 * heads + 6 * kv) * dh < 256 << 20
    g = torch.Generator(device=DEV).manual_seed(86)
    x = torch.randn(n, heads + 2 * kv, dh, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = x.split([heads, kv, kv], dim=1)
    gain = torch.randn(dh, generator=g, device=DEV).to(torch.bfloat16)
    columns = -(-n // page) + 1
    caches = [QuantPagedCache.empty(columns, page, kv, dh, 1, columns, device=DEV) for _ in range(2)]
    for c in caches:
        c.page_table.copy_(torch.randperm(columns, generator=torch.Generator().manual_seed(3))[None])
    seq = torch.zeros(n, dtype=torch.int32, device=DEV)
    slot = torch.arange(7, n + 7, dtype=torch.int32, device=DEV)
    whole = caches[0].append(q, k, v, seq, slot, q_norm=gain, k_norm=gain)
    for a, b in ((0, 4333), (4333, 8600), (8600, n)):
        part = caches[1].append(q[a:b], k[a:b], v[a:b], seq[a:b], slot[a:b], q_norm=gain, k_norm=gain)
        assert torch.equal(whole[a:b], part)
    for name in ("k_pages", "k_scales", "v_pages", "v_scales"):
        assert torch.equal(*(getattr(c, name).view(torch.uint8) for c in caches)), name
    for a, b in zip(*(c.read(seq, slot) for c in caches)):
        assert torch.equal(a, b)
    assert (caches[0].read(seq, slot)[1].float() - v.float()).abs().max() <= 2.0 ** -4 * v.float().abs().max()


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("dh", [64, 128])
def test_append_sizes_and_borders(t, dh):
    """Heads from the type's smallest values to its largest, zeros, a largest magnitude at 448 2^e and its
    neighbours, values half way between codes; no rotation, so keys and values round alike."""
    big = torch.finfo(TYPES[t]).max
    sizes = [0.0, 2.0 ** -24, 2.0 ** -14, 1.0, 448.0, 447.0, 450.0, 224.0, 225.0, 7.0 * 2 ** 10, big, big / 2]
    sizes += [2.0 ** -133, 2.0 ** -126, 2.0 ** -118, 2.0 ** -117, 2.0 ** 100] if t == "bf16" else [61440.0, 63000.0, 57344.0]

    def change(q, k, v):
        for i, s in enumerate(sizes):
            for x in (k, v):
                x[i].clamp_(-3, 3).div_(3).mul_(s)
                x[i, :, i % 5] = s
                x[i, :, 40] = -s / 448 * 3.5 * 2 ** -6   # half way between codes 3 and 4
                x[i, :, 41] = s / 448 * 27               # between 26 and 28
    _append(70, t, 2, 2, dh, 16, [len(sizes)], [(0, j) for j in range(len(sizes))], pairs=(), change=change)


@pytest.mark.parametrize("norm", [False, True])
def test_append_nan_and_infinities(norm):
    """NaN stays where it is, infinities become NaN codes, and neither counts for the scale (a norm carries them through its head)."""
    def change(q, k, v):
        k[3, 0, 5] = float("nan")
        k[4, 1, 60] = float("inf")
        v[5, 0, 0], v[5, 1, 127] = float("-inf"), float("nan")
        v[6, 1] = float("nan")
        k[7, 0] = float("inf")
        q[8, 0, 3] = float("nan")
    _append(71, "bf16", 2, 2, 128, 16, [20], [(0, j) for j in range(20)], pairs=(), norm=norm, change=change)


# --------------------------------------------------------------------- read
def _read(pool, rows, k_out=None, v_out=None):
    k, v = pool.cache.read(pool.ints([s for s, _ in rows]), pool.ints([j for _, j in rows]), k_out=k_out, v_out=v_out)
    val = Values(pool.cache, pool.t)
    assert k.shape == v.shape == (len(rows), pool.kv, pool.dh) and k.dtype == v.dtype == TYPES[pool.t]
    k, v, kw, vw = _np(k), _np(v), val.k_pages.numpy(), val.v_pages.numpy()
    for i, (s, j) in enumerate(rows):
        at = op.place(pool.table, pool.cache.k_pages.shape[0], pool.page, s, j)
        want = (kw[at[0], :, at[1]], vw[at[0], :, :, at[1]]) if at else (np.zeros((pool.kv, pool.dh)),) * 2
        assert np.array_equal(k[i], want[0], equal_nan=True) and np.array_equal(v[i], want[1], equal_nan=True), i


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("kv,dh,page", [(2, 128, 16), (4, 64, 32), (1, 128, 64), (3, 64, 128), (1, 64, 16), (33, 128, 16)])
def test_read_rows(t, kv, dh, page):
    """A prompt, a run that starts and ends inside a page, single rows in any order, the same row several times."""
    pool = Pool(81, t, kv, dh, page, [150, 1, 77])
    r = pool.r
    _read(pool, [(0, j) for j in range(150)] + [(1, 0)] + [(2, j) for j in range(9, 70)])
    _read(pool, [(0, int(j)) for j in r.integers(0, 150, 40)] + [(2, 5)] * 3 + [(2, j) for j in range(76, -1, -3)])
    for n in (1, 2, 15, 16, 17, 63, 64, 65, 79):
        _read(pool, [(0, 3 + j) for j in range(n)])


def test_read_rows_without_a_place_are_zero():
    pool = Pool(82, "bf16", 2, 128, 16, [20, 33, 1])
    _read(pool, [(0, 0), (-1, 0), (0, 1), (3, 0), (2 ** 30, 5), (0, -1), (0, 16 * 20), (0, 17), (1, 3), (1, 60), (-2 ** 31, 2 ** 31 - 1)])
    _read(pool, [(-1, j) for j in range(40)])
    k, v = pool.cache.read(pool.ints([]), pool.ints([]))
    assert k.shape == v.shape == (0, 2, 128)


def test_read_into_given_tensors():
    pool = Pool(83, "fp16", 2, 64, 32, [70])
    wide = torch.full((70, 7, 64), 9.0, dtype=torch.float16, device=DEV)
    _read(pool, [(0, j) for j in range(70)], wide[:, 1:3], wide[:, 4:6])
    assert (wide[:, [0, 3, 6]] == 9).all()


def test_read_keys_or_values_alone():
    """Through the C ABI either output may be missing."""
    from paper_2608_10824_amd import gvc
    pool = Pool(85, "bf16", 2, 128, 16, [100])
    c, n = pool.cache, 100
    seq, slot = pool.ints([0] * n), pool.ints(range(n))
    want = c.read(seq, slot)
    desc = gvc.PagedDesc(gvc.BF16, 2, 2, 128, 16, c.k_pages.shape[0], 1, c.page_table.shape[1])
    for i in range(2):
        got = [torch.full_like(want[0], 7.0) for _ in range(2)]
        p = [got[j].data_ptr() if i == j else None for j in range(2)]
        gvc.quant_read(desc, seq.data_ptr(), slot.data_ptr(), n, *c._pages(), p[0], 256, p[1], 256,
                       torch.cuda.current_stream().cuda_stream)
        assert torch.equal(got[i], want[i]) and (got[1 - i] == 7).all()


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_read_every_code_and_scale(t):
    """All 256 codes under all 256 scales: 2^-127, NaN, values that 16 bits round, and such that pass the type's range."""
    codes = np.arange(256, dtype=np.uint8).reshape(1, 1, 4, 64)
    k = np.broadcast_to(codes, (64, 1, 4, 64)).reshape(16, 1, 16, 64)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 4, 1)   # [scale][quarter]
    table = np.arange(64, dtype=np.int32).reshape(1, 64)
    # slot 4 s + i holds codes 64 i .. 64 i + 63 with scale s
    k = np.broadcast_to(codes.reshape(4, 64), (256, 4, 64)).reshape(64, 1, 16, 64)
    scales = scales.reshape(64, 1, 16)
    pool = Pool.__new__(Pool)
    pool.t, pool.kv, pool.dh, pool.page, pool.table = t, 1, 64, 16, table
    pool.cache = Pool.of(k, scales, k, scales, table, t)
    _read(pool, [(0, j) for j in range(1024)])


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_read_rows_keep_their_values_when_appended_again(t):
    """Into another cache of other pages: the same attention, bit for bit."""
    from paper_2608_10824_amd.paged import PagedCache, QuantPagedCache
    pool = Pool(84, t, 2, 128, 16, [333])
    c, n = pool.cache, 333
    seq, slot = pool.ints([0] * n), pool.ints(range(n))
    k, v = c.read(seq, slot)
    other = QuantPagedCache.empty(6, 64, 2, 128, 1, 6, dtype=TYPES[t], device=DEV)
    other.page_table.copy_(pool.ints([[3, 0, 5, 1, 2, 4]]))
    assert other.append(None, k, v, seq, slot, rope_pairs=()) is None
    for x, y in zip(other.read(seq, slot), (k, v)):
        assert torch.equal(x, y)
    # in 16 bits: the same values, so the same outputs within their bounds
    plain = PagedCache.empty(6, 64, 2, 128, 1, 6, dtype=TYPES[t], device=DEV)
    plain.page_table.copy_(other.page_table)
    plain.append(None, k, v, seq, slot, rope_pairs=())
    q = pool.rows(1, 8, 2.0)
    pool.expect(c.decode(q, pool.ints([n])), q, [0], [n - 1])
    pool.expect(other.decode(q, pool.ints([n])), q, [0], [n - 1])
    pool.expect(plain.decode(q, pool.ints([n])), q, [0], [n - 1])


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
    lengths = [9000, 3, 1, 4777]
    pool = Pool(13, t, 2, dh, page, lengths)
    q = pool.rows(4, 8, 2.0)
    out = pool.cache.decode(q, pool.ints(lengths))
    pool.expect(out, q, range(4), [n - 1 for n in lengths])
    out = pool.cache.decode(q, pool.ints(lengths), window=4500, sinks=70)
    pool.expect(out, q, range(4), [n - 1 for n in lengths], 4500, 70)


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
    ks = pool.bytes()[1]
    for s in range(2):
        for j in range(700):
            ks[pool.table[s, j // 16], 0, j % 16] += (j if s == 0 else 700 - j) // 233
    q = pool.rows(2, 4, 4.0)
    pool.expect(pool.cache.decode(q, pool.ints([700, 700])), q, [0, 1], [699, 699])


def test_decode_lengths_past_the_table_and_below_zero():
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


def test_nan_and_overflow_in_sight():
    """What a row sees comes through: a NaN code, a NaN scale, a value past the type's range (an infinity)."""
    pool = Pool(18, "bf16", 1, 64, 16, [40, 40, 40, 40])
    (k, ks, v, vs), t = pool.bytes(), pool.table
    vs[t[0, 1], 0, 4], v[t[0, 1], 0, :, 4], v[t[0, 1], 0, 3, 4] = 253, 0, 0x7e
    v[t[1, 2], 0, 5, 1] = 0x7f
    k[t[2, 0], 0, 7, 0] = 0xff
    vs[t[3, 0], 0, 9] = 255
    q = pool.rows(4, 2)
    out = pool.cache.decode(q, pool.ints([40] * 4))
    assert torch.isinf(out[0, :, 3]).all() and torch.isnan(out[1, :, 5]).all() and torch.isnan(out[2:]).all()
    pool.expect(out, q, range(4), [39] * 4)


# ------------------------------------------------------------------ prefill
@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv,dh,page", [(4, 4, 128, 16), (8, 2, 128, 64), (14, 2, 64, 16), (3, 1, 128, 128), (40, 1, 64, 32)])
def test_prefill_ragged(t, heads, kv, dh, page):
    """Whole prompts, one row, no row, chunks behind a cached prefix, rows with gaps, rows in falling order."""
    pool = Pool(21, t, kv, dh, page, [150, 1, 40, 260, 97, 66])
    gaps = sorted(pool.r.permutation(97)[:41])
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
    pool = Pool(25, "bf16", 2, 64, 16, [100])
    _ragged(pool, 4, [list(range(80)) + [99] * 20])


def test_prefill_rows_that_see_nothing_and_rows_of_no_sequence():
    pool = Pool(26, "bf16", 2, 64, 16, [50, 50, 50])
    lasts = [-1, 3, -1, 49, -5, -1, -1, 7, 8, 9]
    q = pool.rows(10, 4)
    held = torch.full((10, 4, 64), 768.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints([1, 4, 7, 8]), out=held)
    assert (held[0] == 768).all() and (held[8:] == 768).all()
    pool.expect(out[1:8], q[1:8], [0, 0, 0, 1, 1, 1, 2], lasts[1:8])
    held.fill_(768.0)
    out = pool.cache.prefill(q, pool.ints([9] * 10), pool.ints([4, 2, 5, 99]), out=held)
    assert (held[:2] == 768).all() and not (held[2:] == 768).any()
    pool.expect(out[2:], q[2:], [1] * 3 + [2] * 5, [9] * 8)


def test_values_of_later_slots_do_not_reach_earlier_rows():
    """NaN codes and scales and overflowing values in slots that only later rows see."""
    for window, sinks in ((0, 0), (40, 4)):
        pool = Pool(27, "bf16", 2, 64, 16, [200])
        (k, ks, v, vs), t = pool.bytes(), pool.table
        v[t[0, 5], 0, 3, 7] = 0x7f                                       # slot 87
        vs[t[0, 8], 1, 1], v[t[0, 8], 1, :, 1], v[t[0, 8], 1, 9, 1] = 253, 0, 0x7e   # slot 129: an infinity
        k[t[0, 9], 0, 15, 0] = 0x7f                                      # slot 159
        vs[t[0, 10], 1, 3] = 255                                         # slot 163
        _, out, _, _, _ = _ragged(pool, 4, [range(200)], window, sinks)
        o = _np(out)
        assert np.isfinite(o[:87]).all() and np.isnan(o[87, :2, 3]).all() and np.isfinite(o[:159, 2:, :9]).all()
        assert np.isinf(o[129, 2:, 9]).all() and np.isnan(o[159, :2]).all() and np.isnan(o[163, 2:]).all()


def test_prefill_of_one_row_is_decode():
    pool = Pool(29, "bf16", 2, 128, 16, [37, 600, 1])
    q = pool.rows(3, 8)
    d = pool.cache.decode(q, pool.ints([37, 600, 1]))
    p = pool.cache.prefill(q, pool.ints([36, 599, 0]), pool.ints([0, 1, 2, 3]))
    pool.expect(d, q, range(3), [36, 599, 0])
    pool.expect(p, q, range(3), [36, 599, 0])


# ------------------------------------- prefill: lists long enough for tiles of 128 rows
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
    held = torch.full((n, heads, 64), 768.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints([7, n - 9, n - 6]), out=held)
    assert (held[:7] == 768).all() and (held[n - 6:] == 768).all()
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
    (k, ks, v, vs), tb = pool.bytes(), pool.table
    v[tb[0, 5], 0, 3, 7] = 0x7f                                        # slot 87
    vs[tb[0, 8], 1, 1], v[tb[0, 8], 1, :, 1] = 253 if t == "bf16" else 140, 0
    v[tb[0, 8], 1, 9, 1] = 0x7e                                        # slot 129: an infinity
    k[tb[0, 9], 0, 15, 0] = 0x7f                                       # slot 159
    vs[tb[0, 10], 1, 3] = 255                                          # slot 163
    _tiled(pool, 256, heads, window, sinks)
    _, out, _, _, _ = _ragged(pool, heads, [range(256)], window, sinks)
    o, g = _np(out), heads // 2
    assert np.isfinite(o[:87]).all() and np.isnan(o[87, :g, 3]).all() and np.isfinite(o[:159, g:, :9]).all()
    assert np.isinf(o[129, g:, 9]).all() and np.isnan(o[159, :g]).all() and np.isnan(o[163, g:]).all()
    if window:
        assert np.isfinite(o[203:]).all()


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_tiles_of_steep_scores(t):
    """The running maximum moves up and down over hundreds."""
    pool = Pool(58, t, 1, 64, 16, [256])
    ks = pool.bytes()[1]
    for j in range(256):
        ks[pool.table[0, j // 16], 0, j % 16] += j % 50 // 17
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
    want = pool.cache.prefill(q, pool.ints(range(256)), pool.ints([0, 256]), scale=0.3)
    assert torch.equal(pool.cache.prefill(q, pool.ints(range(256)), pool.ints([0, 256]), scale=0.3, out=q), want)


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


@pytest.mark.parametrize("rows,length", [(10, 50), (10, 3000), (300, 3000), (400, 3000)])
def test_prefill_with_bounds_that_fall(rows, length):
    """Bounds have to rise; where they do not, no row outside them is touched (nor any other memory)."""
    pool = Pool(26, "bf16", 2, 64, 16, [length] * 4)
    q = pool.rows(rows + 9, 4)
    held = torch.full((rows + 9, 4, 64), 768.0, dtype=torch.bfloat16, device=DEV)
    pool.cache.prefill(q, pool.ints([length - 1] * (rows + 9)), pool.ints([0, rows, 0, rows, rows + 7]), out=held)
    assert (held[rows + 7:] == 768).all()


# ------------------------------------------------------- workspaces of split calls
def test_a_workspace_may_hold_anything():
    """Split decodes and prefills through the C ABI, in memory that holds zeros,
    ones, noise, another call's rest and their own: the same bits."""
    from paper_2608_10824_amd import gvc
    pool = Pool(61, "bf16", 2, 128, 16, [7000, 17, 2100, 0])
    c = pool.cache
    desc = gvc.PagedDesc(gvc.BF16, 8, 2, 128, 16, c.k_pages.shape[0], 4, c.page_table.shape[1])
    q, lengths, begin = pool.rows(20, 8), pool.ints([7000, 17, 2100, 0]), pool.ints([0, 1, 2, 20, 20])
    last = pool.ints([6999, 16] + list(range(2082, 2100)))
    long_q, long_last, long_begin = pool.rows(300, 8), pool.ints(range(1800, 2100)), pool.ints([0, 0, 0, 300, 300])
    pages = c._pages()
    sizes = [gvc.quant_workspace(desc, False, 4), gvc.quant_workspace(desc, True, 20), gvc.quant_workspace(desc, True, 300)]
    assert min(sizes) > 0
    work = torch.zeros(max(sizes), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream

    def run():
        outs = [torch.empty_like(x) for x in (q[:4], q, long_q)]
        gvc.quant_decode(desc, 0.09, 0, 0, q.data_ptr(), 1024, lengths.data_ptr(), *pages, outs[0].data_ptr(), 1024,
                         work.data_ptr(), sizes[0], stream)
        gvc.quant_prefill(desc, 0.09, 0, 0, q.data_ptr(), 1024, last.data_ptr(), begin.data_ptr(), 20, *pages,
                          outs[1].data_ptr(), 1024, work.data_ptr(), sizes[1], stream)
        gvc.quant_prefill(desc, 0.09, 0, 0, long_q.data_ptr(), 1024, long_last.data_ptr(), long_begin.data_ptr(), 300,
                          *pages, outs[2].data_ptr(), 1024, work.data_ptr(), sizes[2], stream)
        return outs

    want = run()
    pool.expect(want[0], q[:4], range(4), [6999, 16, 2099, -1], scale=0.09)
    pool.expect(want[1], q, [0, 1] + [2] * 18, [6999, 16] + list(range(2082, 2100)), scale=0.09)
    noise = torch.randint(0, 256, work.shape, dtype=torch.uint8, device=DEV)
    for fill in (None, 255, 1, noise):
        if fill is not None:
            work.copy_(noise) if fill is noise else work.fill_(fill)
        for x, y in zip(want, run()):
            assert torch.equal(x, y)


# ------------------------------------------- values near the end of the type's range
def _large(pool, power):
    """The pool's values up to 2^(power + 3), all of one sign: their sums before the division are larger."""
    v, vs = pool.bytes()[2:]
    v.copy_(torch.where((v & 127) == 127, v, v & 127))
    held = vs != 255
    vs[held] = vs[held].clamp(max=119) + power   # 448 2^-8 times 2^power at most


@pytest.mark.parametrize("power", [90, 114, 121, 126])
def test_outputs_are_finite_where_sums_overflow(power):
    """bf16 values to 2^127: decode (split and not, with a window) and lists of few rows give
    the finite outputs of their formulas."""
    lengths = [1, 40, 700, 6000, 0]
    pool = Pool(63, "bf16", 2, 64, 16, lengths)
    _large(pool, power)
    q = pool.rows(5, 8, 2.0)
    pool.expect(pool.cache.decode(q, pool.ints(lengths)), q, range(5), [n - 1 for n in lengths])
    pool.expect(pool.cache.decode(q, pool.ints(lengths), window=300, sinks=20), q, range(5), [n - 1 for n in lengths], 300, 20)
    _ragged(pool, 8, [[0], range(40), [699, 3], [5999], []])


@pytest.mark.parametrize("power", [90, 114, 121, 126])
@pytest.mark.parametrize("dh,heads,columns", [(64, 72, 0), (128, 72, 0), (64, 6, 200), (128, 6, 200)])
def test_tiles_are_finite_where_sums_overflow(power, dh, heads, columns):
    pool = Pool(65, "bf16", 2, dh, 16, [256], extra_columns=columns)
    _large(pool, power)
    _tiled(pool, 256, heads)
    _ragged(pool, heads, [range(256)])


# ------------------------- calls of many sequences and many heads, by the path that they take
@pytest.mark.parametrize("seqs,heads,kv", [(64, 4, 2), (65, 6, 2), (130, 2, 1)])
def test_decode_many_sequences(seqs, heads, kv):
    """Ragged batches of 64 sequences and more, idle ones among them; rows of the same as a prefill."""
    r = np.random.default_rng(41)
    lengths = [int(n) for n in np.where(r.random(seqs) < 0.2, 0, np.exp(r.uniform(0, 7.7, seqs)))]
    pool = Pool(41, "bf16", kv, 64, 16, lengths)
    q = pool.rows(seqs, heads)
    out = pool.cache.decode(q, pool.ints(lengths))
    pool.expect(out, q, range(seqs), [n - 1 for n in lengths])
    out = pool.cache.decode(q, pool.ints(lengths), window=333, sinks=20)
    pool.expect(out, q, range(seqs), [n - 1 for n in lengths], 333, 20)
    if seqs * kv <= 130:
        rows = [[n - 1, n // 2][:int(r.integers(0, 3))] if n else [] for n in lengths]
        _ragged(pool, heads, rows)


@pytest.mark.parametrize("seqs,kv,length", [(64, 8, 60000), (70, 2, 30000), (3, 8, 140000)])
def test_decode_long_sequences_on_the_same_pages(seqs, kv, length):
    """Lengths at which chunks are hundreds of tiles; all tables name the pages of one small pool."""
    page, n_pages = 128, 40
    pool = Pool(42, "fp16", kv, 64, page, [page * n_pages], spare=0, extra_columns=0)
    columns = -(-length // page)
    pool.table = pool.r.integers(0, n_pages, (seqs, columns)).astype(np.int32)
    c = pool.cache
    pool.cache = c = type(c)(c.k_pages, c.k_scales, c.v_pages, c.v_scales, torch.tensor(pool.table, device=DEV), TYPES["fp16"])
    lengths = [int(length * f) for f in np.linspace(0.6, 1, seqs)]
    lengths[1] = 5
    q = pool.rows(seqs, kv)
    out = c.decode(q, pool.ints(lengths))
    pick = [0, 1, seqs // 2, seqs - 1]
    pool.expect(out[pick], q[pick], pick, [lengths[i] - 1 for i in pick])


@pytest.mark.parametrize("t,dh,heads,kv", [("bf16", 64, 32, 32), ("fp16", 64, 64, 32), ("bf16", 128, 34, 34)])
def test_units_of_many_heads_join_long_chunks_themselves(t, dh, heads, kv):
    """4200 to 16384 slots of at least 32 key-value heads: eight long chunks and no second launch."""
    lengths = [5400, 300, 0, 4300]
    pool = Pool(71, t, kv, dh, 16, lengths, extra_columns=600)
    q = pool.rows(4, heads, 2.0)
    for _ in range(2):   # the second in memory that the first has left
        pool.expect(pool.cache.decode(q, pool.ints(lengths)), q, range(4), [n - 1 for n in lengths])
    pool.expect(pool.cache.decode(q, pool.ints(lengths), window=4400, sinks=40), q, range(4), [n - 1 for n in lengths], 4400, 40)
    if 4 * kv <= 128:
        _ragged(pool, heads, [range(5390, 5400), [299, 0], [], [4299]])


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
    held = torch.full((n, heads, 64), 768.0, dtype=torch.bfloat16, device=DEV)
    out = pool.cache.prefill(q, pool.ints(lasts), pool.ints(begin), out=held)
    assert (held[:3] == 768).all() and (held[n - 5:] == 768).all()
    pick = sorted({x for s in range(seqs) for x in (begin[s], begin[s + 1] - 1) if begin[s + 1] > begin[s]})
    pool.expect(out[pick], q[pick], [seq[i] for i in pick], [lasts[i] for i in pick])


@pytest.mark.parametrize("length", [3000, 6000])
def test_few_rows_of_many_sequences(length):
    """Lists of few rows in 70 sequences, joined by their units and by a second launch, which looks a row's sequence up."""
    r = np.random.default_rng(74)
    lengths = [int(n) for n in r.integers(1, 100, 70)]
    lengths[3], lengths[66] = length, length - 400
    pool = Pool(74, "bf16", 1, 64, 16, lengths)
    rows = [[n - 1] if s % 3 else [] for s, n in enumerate(lengths)]
    rows[3], rows[66], rows[69] = [length - 1, 7], [length - 401, length - 402, 900], [0]
    assert sum(len(x) for x in rows) * 8 <= 70 * 16
    _ragged(pool, 8, rows)


# ----------------------------------------------------------------- together
def test_a_history_appended_attended_and_moved():
    """Two sequences from an empty cache: a prompt, a second chunk, then single
    tokens; each step's attention over what has been appended so far; in the end one moves to a 16-bit cache."""
    from paper_2608_10824_amd.paged import PagedCache, QuantPagedCache
    heads, kv, dh, page = 6, 2, 128, 16
    c = QuantPagedCache.empty(30, page, kv, dh, 2, 12, device=DEV)
    assert (c.page_table == -1).all()
    ids = np.random.default_rng(31).permutation(30)[:24].reshape(2, 12).astype(np.int32)
    c.page_table.copy_(torch.tensor(ids))
    pool = Pool.__new__(Pool)
    pool.r, pool.t, pool.kv, pool.dh, pool.page, pool.cache, pool.table = np.random.default_rng(32), "bf16", kv, dh, page, c, ids
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
        v = _np(x[:, heads + kv:])
        _, got = c.read(seq, slot)   # within half a step of what was appended
        most = np.abs(v).max(-1, keepdims=True)
        assert (np.abs(_np(got) - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * most / 224)).all()
        have = [have[s] + new[s] for s in range(2)]
        if max(new) > 1:
            out = c.prefill(q, slot, pool.ints([0, new[0], new[0] + new[1]]), window=50, sinks=4)
            pool.expect(out, q, [s for s, _ in rows], [j for _, j in rows], 50, 4)
        elif min(new) == 1:
            out = c.decode(q, pool.ints(have), window=50, sinks=4)
            pool.expect(out, q, [0, 1], [have[0] - 1, have[1] - 1], 50, 4)
    k, v = c.read(pool.ints([1] * have[1]), pool.ints(range(have[1])))
    plain = PagedCache.empty(8, page, kv, dh, 1, 8, device=DEV)
    plain.page_table.copy_(pool.ints([range(8)]))
    plain.append(None, k, v, pool.ints([0] * have[1]), pool.ints(range(have[1])), rope_pairs=())
    q = pool.rows(1, heads)
    pool.expect(plain.decode(q, pool.ints(have[1:])), q, [1], [have[1] - 1])


def test_captured_calls_replay_beside_eager_ones():
    """One graph of append, decode, prefill and read, replayed with new inputs and a
    changed table, eager calls and a second graph's replays between: each
    replay is bit for bit the eager result."""
    pool = Pool(33, "bf16", 2, 64, 16, [90, 1500, 1], spare=60)
    c = pool.cache
    q, k, v = pool.rows(3, 8), pool.rows(3, 2), pool.rows(3, 2)
    seq, slot, lengths = pool.ints([0, 1, 2]), pool.ints([89, 1499, 0]), pool.ints([90, 1500, 1])
    last, begin = pool.ints([89, 1499, 0]), pool.ints([0, 1, 2, 3])

    def step():
        r = c.append(q, k, v, seq, slot)
        return (r, c.decode(r, lengths), c.prefill(r, last, begin, window=64, sinks=3)) + c.read(seq, slot)

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
        slot.copy_(pool.ints([89, 1499 - turn, 0]))
        lengths.copy_(pool.ints([90 - turn, 1500, turn % 2]))
        if turn == 2:   # the second sequence's first page moves
            for x in pool.bytes():
                x[spare[0]] = x[int(pool.table[1, 0])]
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
    pool = Pool(34, "bf16", 2, 128, 16, [3000, 40])
    c = pool.cache
    lengths = pool.ints([3000, 40])
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


def test_outputs_in_place_of_their_inputs():
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
    want = c.prefill(q, slot, pool.ints([0, n, n, n]))
    assert torch.equal(c.prefill(q, slot, pool.ints([0, n, n, n]), out=q), want)


def test_pool_over_four_gib():
    """Pages whose byte offsets pass 32 bits."""
    from paper_2608_10824_amd.paged import QuantPagedCache
    kv, dh, page, n_pages = 8, 128, 128, 35000   # 4.3 GiB each of keys and values
    c = QuantPagedCache.empty(n_pages, page, kv, dh, 2, 4, device=DEV)
    pages = np.array([[n_pages - 1, 3, n_pages - 2, 16400], [1, n_pages - 3, 2, 0]], dtype=np.int32)
    c.page_table.copy_(torch.tensor(pages))
    g = torch.Generator(device=DEV).manual_seed(35)
    n = 400
    x = torch.randn(n, 32, dh, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = x[:, :16], x[:, 16:24], x[:, 24:]
    seq = torch.tensor([i % 2 for i in range(n)], dtype=torch.int32, device=DEV)
    slot = torch.tensor([i // 2 for i in range(n)], dtype=torch.int32, device=DEV) + 200
    assert torch.equal(c.append(q, k, v, seq, slot, rope_pairs=()), q)
    # a small pool with the same pages gives the same rows and the same attention
    at = torch.tensor(pages.flatten().astype(np.int64), device=DEV)
    small = QuantPagedCache(*(y.view(torch.uint8)[at].view(y.dtype) for y in (c.k_pages, c.k_scales, c.v_pages, c.v_scales)),
                            torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4))
    for got, same, want in zip(c.read(seq, slot), small.read(seq, slot), (k, v)):
        assert torch.equal(got, same) and (got.float() - want.float()).abs().max() < 0.3
    qd = q[:2].contiguous()
    lengths = torch.tensor([400, 399], dtype=torch.int32, device=DEV)
    assert torch.equal(c.decode(qd, lengths), small.decode(qd, lengths))
    last = torch.tensor([399, 120, 399], dtype=torch.int32, device=DEV)
    begin = torch.tensor([0, 2, 3], dtype=torch.int32, device=DEV)
    qp = q[:3].contiguous()
    assert torch.equal(c.prefill(qp, last, begin), small.prefill(qp, last, begin))


@pytest.mark.parametrize("t,size", [("bf16", 124), ("fp16", 13)])
@pytest.mark.parametrize("dh", [64, 128])
def test_heads_below_the_types_normal_range(t, size, dh):
    """Keys and values that the type holds with few bits (rounded, some to zero), under queries and a scale
    that make their scores count.  Outputs in bf16 are as small: rounded to steps of 2^-133 (off by 2^-134), of a sum
    in 32 bits whose 300 products and divisions are rounded to steps of 2^-149 (off by 600 * 2^-150 in all, for a sum of
    weights of 1 or more), which is less than 2^-133 together.  (The fp16 bounds hold fp16's steps already.)"""
    least = 2.0 ** -133 if t == "bf16" else 0.0
    pool = Pool(81, t, 2, dh, 16, [300, 40])
    k, ks, v, vs = pool.bytes()
    low = 1 if t == "bf16" else 103   # 2^-126, 2^-24
    for x in (ks, vs):
        x.copy_(torch.tensor(pool.r.integers(low, low + 4, tuple(x.shape)).astype(np.uint8)))
    for x in (k, v):
        x.copy_(torch.tensor(pool.r.integers(0, 0x48, tuple(x.shape)).astype(np.uint8)))
    q = pool.rows(2, 4, 2.0 ** size)
    pool.expect(pool.cache.decode(q, pool.ints([300, 40]), scale=64.0), q, [0, 1], [299, 39], scale=64.0, least=least)
    rows = [(0, j) for j in range(200, 300)] + [(1, j) for j in range(40)]
    for heads in (4, 20):
        q = pool.rows(140, heads, 2.0 ** size)
        out = pool.cache.prefill(q, pool.ints([j for _, j in rows]), pool.ints([0, 100, 140]), scale=64.0)
        pool.expect(out, q, [s for s, _ in rows], [j for _, j in rows], scale=64.0, least=least)


@pytest.mark.parametrize("dh", [64, 128])
def test_nan_and_overflow_in_sight_of_fp16(dh):
    """A NaN code, a NaN scale and values past the type's range, seen by some rows."""
    pool = Pool(82, "fp16", 1, dh, 16, [40] * 4)
    (k, ks, v, vs), t = pool.bytes(), pool.table
    vs[t[0, 1], 0, 4], v[t[0, 1], 0, :, 4], v[t[0, 1], 0, 3, 4] = 135, 0, 0x7e   # 448 * 2^8
    v[t[1, 2], 0, 5, 1] = 0x7f
    k[t[2, 0], 0, 7, 0] = 0xff
    vs[t[3, 0], 0, 9] = 255
    q = pool.rows(4, 2)
    out = pool.cache.decode(q, pool.ints([40] * 4))
    assert torch.isinf(out[0, :, 3]).all() and torch.isnan(out[1, :, 5]).all() and torch.isnan(out[2:]).all()
    pool.expect(out, q, range(4), [39] * 4)
    lasts = [j for _ in range(4) for j in range(40)]
    for heads in (2, 60):
        q = pool.rows(160, heads)
        out = pool.cache.prefill(q, pool.ints(lasts), pool.ints([0, 40, 80, 120, 160]))
        assert torch.isinf(out[20:40, :, 3]).all() and torch.isfinite(out[:20]).all()
        pool.expect(out, q, [s for s in range(4) for _ in range(40)], lasts)


# --------------------------------------------------- append at the ends of 32 bits
def _keys(pool, k, positions, pairs=None, gain=None, eps=1e-5):
    """Appends keys k [rows][kv][dh] to sequence 0 from slot 0 on; their codes and scales have to be the exact keys', bit for bit."""
    c, n = pool.cache, k.shape[0]
    c.append(None, k, k, pool.ints([0] * n), pool.ints(range(n)), positions=positions and pool.ints([positions]), rope_pairs=pairs,
             k_norm=gain, rms_eps=eps)
    pairs = (pool.dh // 2,) if pairs is None else pairs
    x, g = _np(k), None if gain is None else _np(gain)
    want = np.array([[op.rope_norm(x[i, h], positions and [positions[i]], pairs, 1e4, g, eps) for h in range(pool.kv)] for i in range(n)])
    assert np.isfinite(want).all()
    codes, scales = oq.quantise_heads(want, pool.t)
    got = pool.bytes()
    at = [op.place(pool.table, c.k_pages.shape[0], pool.page, 0, j) for j in range(n)]
    page, off = (np.array(x) for x in zip(*at))
    assert np.array_equal(got[1].cpu().numpy()[page, :, off], scales)
    wrong = got[0].cpu().numpy()[page, :, off] != codes
    assert not wrong.any(), "%d of %d codes, first %s" % (wrong.sum(), wrong.size, np.argwhere(wrong)[0])
    return want


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("norm", [False, True])
def test_append_finite_keys_past_the_largest_float(dh, norm):
    """Rotation, or a gain, carries finite values past what 32 bits hold: they become the largest code, not NaN."""
    pool = Pool(87, "bf16", 2, dh, 16, [40])
    big = torch.finfo(torch.bfloat16).max
    k = torch.tensor(pool.r.choice([-1.0, 1.0], (40, 2, dh)) * pool.r.uniform(0.5, 1, (40, 2, dh)) * big).to(torch.bfloat16)
    gain = None
    if norm:
        k = pool.rows(40, 2)
        gain = torch.tensor(pool.r.uniform(0.5, 1, dh) * big).to(torch.bfloat16).to(DEV)
    want = _keys(pool, k.to(DEV), [17 * j for j in range(40)], gain=gain)
    assert (np.abs(want) > 2.0 ** 128).any()


@pytest.mark.parametrize("dh", [64, 128])
def test_append_keys_below_the_smallest_normal_float(dh):
    """Keys of about 2^-130, which 32 bits hold in steps of 2^-149: one in some tens of thousands is so near to half
    way between two codes that it would be half way after a rounding to them."""
    pool = Pool(88, "bf16", 8, dh, 16, [300])
    gain = torch.tensor(pool.r.uniform(0.5, 1, dh) * 2.0 ** -129).to(torch.bfloat16).to(DEV)
    want = _keys(pool, pool.rows(300, 8), None, pairs=(), gain=gain)
    assert np.abs(want).max() < 2.0 ** -126


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_append_norms_whose_squares_leave_32_bits(dh, eps):
    """Heads of which a square, or the sum of them, is past the largest float, or (without rms_eps) below the smallest."""
    powers = [0, 40, 62, 63, 64, 65, 100, 125] if eps else [-30, -50, -62, -75, -100, -120]

    def change(q, k, v):
        for i, p in enumerate(powers):
            q[i] *= 2.0 ** p
            k[i] *= 2.0 ** p
    _append(89, "bf16", 8, 2, dh, 16, [20], [(0, j) for j in range(12)], norm=True, eps=eps, change=change)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_append_queries_keep_nan_and_infinities(t, norm):
    """A query's NaN and infinities come out where the formula has them: in place without a norm, in the partner too
    where the pair turns, through the whole head with a norm."""
    heads, dh, n = 3, 128, 6
    pool = Pool(90, t, 1, dh, 16, [n])
    q, k = pool.rows(n, heads), pool.rows(n, 1)
    q[1, 0, 3], q[2, 1, 100], q[3, 2, 5], q[4, 0, 70] = (float(x) for x in ("nan", "nan", "inf", "-inf"))
    gain = torch.tensor(1 + 0.2 * pool.r.standard_normal(dh)).to(TYPES[t]).to(DEV) if norm else None
    out = _np(pool.cache.append(q, k, k, pool.ints([0] * n), pool.ints(range(n)), rope_pairs=(32,), q_norm=gain))
    x, u = _np(q), _u(t)
    for i in range(n):
        for h in range(heads):
            with np.errstate(invalid="ignore"):
                want = op.rope_norm(x[i, h], [i], (32,), 1e4, None if gain is None else _np(gain), 1e-5)
            fine = np.isfinite(want)
            assert np.array_equal(np.isnan(out[i, h]), np.isnan(want)), (i, h)
            inf = np.isinf(want)
            assert np.array_equal(out[i, h][inf], want[inf]), (i, h)
            mag = 2 * np.abs(want[fine]).max(initial=0)   # at least |x| + |y| of any pair
            with np.errstate(invalid="ignore"):
                off = np.abs(out[i, h] - want) - u * np.abs(want) - mag * (2.0 ** -20 + 136 * 2.0 ** -24) * (1 + u) - _tiny(t)
            assert off[fine].max(initial=0) <= 0, (i, h)
    assert np.isnan(out[1, 0]).any() and np.isnan(out[2, 1]).any()


@pytest.mark.parametrize("t,dh", [("bf16", 64), ("fp16", 64), ("fp16", 128)])
def test_a_long_append_of_other_types_is_its_parts(t, dh):
    """As above for the other types and heads, with rows that skip slots and rows of no sequence."""
    from paper_2608_10824_amd.paged import QuantPagedCache
    heads, kv, page, n = 32, 8, 64, 26000 if dh == 64 else 13000
    assert n * (4 * heads + 6 * kv) * dh > 256 << 20 and n // 2 * (4 * heads + 6 * kv) * dh < 256 << 20
    g = torch.Generator(device=DEV).manual_seed(91)
    q, k, v = torch.randn(n, heads + 2 * kv, dh, generator=g, device=DEV).to(TYPES[t]).split([heads, kv, kv], dim=1)
    gain = torch.randn(dh, generator=g, device=DEV).to(TYPES[t])
    columns = n * 9 // 8 // page + 1
    caches = [QuantPagedCache.empty(columns, page, kv, dh, 1, columns, dtype=TYPES[t], device=DEV) for _ in range(2)]
    for c in caches:
        c.page_table.copy_(torch.randperm(columns, generator=torch.Generator().manual_seed(4))[None])
    at = torch.arange(n, device=DEV)
    slot = (at * 9 // 8).int()
    seq = torch.where(at % 1001 == 1000, -1, 0).int()
    whole = caches[0].append(q, k, v, seq, slot, q_norm=gain, k_norm=gain)
    for a, b in ((0, n // 2), (n // 2, n)):
        part = caches[1].append(q[a:b], k[a:b], v[a:b], seq[a:b], slot[a:b], q_norm=gain, k_norm=gain)
        assert torch.equal(whole[a:b], part)
    for name in ("k_pages", "k_scales", "v_pages", "v_scales"):
        assert torch.equal(*(getattr(c, name).view(torch.uint8) for c in caches)), name
    assert (caches[0].k_pages.view(torch.uint8) != 0).any() and (caches[0].v_pages.view(torch.uint8) != 0).any()
