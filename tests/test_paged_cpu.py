"""The paged cache on the host: refusals of the C ABI (nothing is launched, so
no GPU is needed), the check of page tables and row lists, and pins of the
oracle that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

from oracle import paged as op
from oracle.llama import attend_row, rope_row


def _desc(**kw):
    from paper_2608_10824_amd import gvc
    d = gvc.PagedDesc(gvc.BF16, 8, 2, 64, 16, 4, 2, 3)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _rope(pairs=(32, 0, 0), theta=1e4, eps=1e-5):
    from paper_2608_10824_amd import gvc
    return gvc.PagedRope((ctypes.c_int32 * 3)(*pairs), theta, eps, None, None, None, 0)


P = 1 << 12   # an aligned address that nothing reads: every call below is refused


def _append(desc, rope, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(q=P, qs=512, k=P, ks=128, v=P, vs=128, row_seq=P, row_slot=P, n=5, kp=P, vp=P, table=P, o=P, os=512)
    a.update(kw)
    gvc.paged_append(desc, rope, *a.values(), None)


def _decode(desc, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(scale=0.125, window=0, sinks=0, q=P, qs=512, lengths=P, kp=P, vp=P, table=P, o=P, os=512, work=None, size=0)
    a.update(kw)
    gvc.paged_decode(desc, *a.values(), None)


def _prefill(desc, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(scale=0.125, window=0, sinks=0, q=P, qs=512, last=P, begin=P, n=5, kp=P, vp=P, table=P, o=P, os=512,
             work=None, size=0)
    a.update(kw)
    gvc.paged_prefill(desc, *a.values(), None)


def _refused(f, *a, code=None, **kw):
    from paper_2608_10824_amd import gvc
    with pytest.raises(gvc.GvcError) as e:
        f(*a, **kw)
    assert e.value.code == (gvc.GVC_EINVAL if code is None else code) and gvc.last_error()


@pytest.mark.parametrize("field,value", [("dtype", 2), ("dtype", -1), ("n_heads", 0), ("n_heads", 7), ("n_heads", 1026),
                                         ("n_kv_heads", 0), ("n_kv_heads", 3), ("head_dim", 96), ("head_dim", 256),
                                         ("page_size", 8), ("page_size", 24), ("page_size", 256), ("n_pages", 0),
                                         ("n_seqs", 0), ("n_seqs", 4097), ("max_pages", 0), ("max_pages", 1 << 27)])
def test_bad_shapes_refused(field, value):
    from paper_2608_10824_amd import gvc
    d = _desc(**{field: value})
    _refused(_append, d, _rope())
    _refused(_decode, d)
    _refused(_prefill, d)
    _refused(gvc.paged_workspace, d, False, 1)


@pytest.mark.parametrize("rope", [dict(pairs=(-4, 8, 0)), dict(pairs=(30, 0, 0)), dict(pairs=(16, 16, 4)),
                                  dict(theta=0.0), dict(theta=-1.0), dict(theta=float("inf")), dict(theta=float("nan")),
                                  dict(eps=-1e-5), dict(eps=float("nan"))])
def test_bad_rotation_refused(rope):
    _refused(_append, _desc(), _rope(**rope))


def test_the_base_keeps_its_64_bits_within_the_range_of_a_float():
    base = 10000 * 8 ** (128 / 126)
    assert _rope(theta=base).theta == base
    for theta in (1e39, -1e39, 1e-46, 1e-320):
        _refused(_append, _desc(), _rope(theta=theta))
    _append(_desc(), _rope(theta=3e38), n=0)
    _append(_desc(), _rope(theta=1e-38), n=0)


@pytest.mark.parametrize("kw", [dict(q=None), dict(o=None), dict(k=None), dict(v=None), dict(row_seq=None),
                                dict(row_slot=None), dict(kp=None), dict(vp=None), dict(table=None), dict(n=-1),
                                dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(o=P + 8), dict(qs=516), dict(ks=120),
                                dict(vs=(1 << 32) + 8), dict(os=0), dict(kp=P + 8), dict(n=1 << 30)])
def test_bad_append_refused(kw):
    _refused(_append, _desc(), _rope(), **kw)


@pytest.mark.parametrize("heads,kv,n", [(1, 1, 1 << 26), (1, 1, 59645042), (2, 1, (1 << 26) - 1), (2, 1, 59645042)])
def test_more_rows_than_a_launch_has_threads_refused(heads, kv, n):
    """n (heads + 2 kv) is below 2^28, but a row takes 64 threads and its values 8: 2^32 are the most."""
    assert n * (heads + 2 * kv) < 1 << 28 and n * (64 + 8 * kv) >= 2 ** 32 - 2 ** 19
    _refused(_append, _desc(n_heads=heads, n_kv_heads=kv), _rope(), n=n, qs=128)


@pytest.mark.parametrize("call", [_decode, _prefill])
@pytest.mark.parametrize("kw", [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
                                dict(window=-1), dict(sinks=-1), dict(q=None), dict(kp=None), dict(vp=None),
                                dict(table=None), dict(o=None), dict(q=P + 8), dict(o=P + 2), dict(vp=P + 2),
                                dict(qs=508), dict(os=448)])
def test_bad_attention_refused(call, kw):
    _refused(call, _desc(), **kw)


def test_bad_lists_refused():
    _refused(_decode, _desc(), lengths=None)
    _refused(_prefill, _desc(), last=None)
    _refused(_prefill, _desc(), begin=None)
    _refused(_prefill, _desc(), n=-1)
    _refused(_prefill, _desc(), n=1 << 27)


def test_largest_tables():
    """2^30 slots in a row of the table and 2^27 entries in all are the most."""
    from paper_2608_10824_amd import gvc
    assert gvc.paged_workspace(_desc(n_seqs=4096, max_pages=1 << 15), False, 4096) > 0
    assert gvc.paged_workspace(_desc(n_seqs=1, max_pages=1 << 26), False, 1) > 0
    _refused(gvc.paged_workspace, _desc(n_seqs=4096, max_pages=(1 << 15) + 1), False, 4096)
    _refused(gvc.paged_workspace, _desc(n_seqs=1, max_pages=(1 << 26) + 1), False, 1)


def test_norm_gains_and_positions_refused():
    r = _rope()
    r.q_norm = P + 2
    _refused(_append, _desc(), r)
    r = _rope()
    r.positions, r.position_stride = P, 4   # five rows
    _refused(_append, _desc(), r)


def test_no_rows_is_nothing_to_do():
    _append(_desc(), _rope(), n=0, q=None, o=None, k=None, v=None, row_seq=None)
    _prefill(_desc(), n=0, q=None, o=None, last=None, begin=None)


def _check(table, lengths=None, seq=(), slot=(), **kw):
    from paper_2608_10824_amd import gvc
    a = [np.ascontiguousarray(x, dtype=np.int32) for x in (table, [] if lengths is None else lengths, seq, slot)]
    p = [x.ctypes.data_as(ctypes.c_void_p).value for x in a]
    gvc.paged_check(_desc(**kw), p[0], None if lengths is None else p[1], p[2], p[3], len(a[2]))


TABLE = [[3, 0, -1], [1, 7, 2]]   # page 7 of 4 and entry -1 are no pages


def test_check_accepts_what_exists():
    _check(TABLE, [32, 16])
    _check(TABLE, [0, 0], [0, 0, 1, -1, 1], [0, 31, 15, 99, 47])
    _check([[3, 0, 1], [3, 2, 1]], [48, 48])   # a page of two sequences is read by both


@pytest.mark.parametrize("lengths,seq,slot,text", [
    ([33, 0], (), (), "sequence 0"), ([0, 17], (), (), "sequence 1"), ([0, 49], (), (), "length 49"),
    ([-1, 0], (), (), "length -1"), (None, [0, 2], [0, 0], "row 1"), (None, [-2], [0], "row 0"),
    (None, [0, 0, 0], [0, 1, 48], "row 2"), (None, [1], [-1], "row 0"), (None, [0, 0], [0, 32], "row 1"),
    (None, [1], [16], "page 7"), (None, [0, 1, 0], [5, 5, 5], "row 2")])
def test_check_names_the_first_fault(lengths, seq, slot, text):
    from paper_2608_10824_amd import gvc
    with pytest.raises(gvc.GvcError) as e:
        _check(TABLE, lengths, seq, slot)
    assert e.value.code == gvc.GVC_EINVAL and text in str(e.value)


def test_check_finds_rows_that_meet_on_a_shared_page():
    _refused(_check, [[3, 0, 1], [3, 2, 1]], None, [0, 1], [7, 7])
    _check([[3, 0, 1], [3, 2, 1]], None, [0, 1], [23, 23])


def test_cache_refuses_host_tensors():
    import torch
    from paper_2608_10824_amd.paged import PagedCache
    k, v = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, 16, dtype=torch.bfloat16)
    table = torch.zeros(2, 3, dtype=torch.int32)
    for a in ((k, v, table), (k.float(), v.float(), table), (k, k, table), (k[0], v[0], table), (k, v, table.long()),
              (k, v.half(), table)):
        with pytest.raises(ValueError):
            PagedCache(*a)


def _host_cache():
    """A cache over host memory, which only __init__ refuses: what its calls check comes before the C call."""
    import torch
    from paper_2608_10824_amd.paged import PagedCache
    c = PagedCache.__new__(PagedCache)
    c.k_pages, c.v_pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, 16, dtype=torch.bfloat16)
    c.page_table = torch.zeros(2, 3, dtype=torch.int32)
    c.n_seqs, c.n_kv_heads, c.head_dim, c._dtype, c._index = 2, 2, 64, torch.bfloat16, -1
    c._shape, c._descs, c._sizes = (c._dtype, 4, 2, 16, 64, 2, 3), {}, {}
    return c


def test_forward_mode_duals_are_refused():
    import torch
    from torch.autograd import forward_ad
    from paper_2608_10824_amd.paged import PagedCache
    c = _host_cache()
    q, k, gain = torch.ones(2, 4, 64, dtype=torch.bfloat16), torch.ones(2, 2, 64, dtype=torch.bfloat16), torch.ones(64).bfloat16()
    two, three = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with forward_ad.dual_level():
        dq, dk, dg = (forward_ad.make_dual(x, x.clone()) for x in (q, k, gain))
        for f in (lambda: c.decode(dq, two), lambda: c.decode(q, two, out=dq), lambda: c.prefill(dq, two, three),
                  lambda: c.prefill(q, two, three, out=dq), lambda: c.append(dq, k, k, two, two),
                  lambda: c.append(q, dk, k, two, two), lambda: c.append(None, k, dk, two, two),
                  lambda: c.append(q, k, k, two, two, q_norm=dg), lambda: c.append(q, k, k, two, two, k_norm=dg),
                  lambda: c.append(q, k, k, two, two, q_out=dq),
                  lambda: PagedCache(forward_ad.make_dual(c.k_pages, c.k_pages.clone()), c.v_pages, c.page_table),
                  lambda: PagedCache(c.k_pages, forward_ad.make_dual(c.v_pages, c.v_pages.clone()), c.page_table)):
            with pytest.raises(ValueError, match="tangent"):
                f()
        with pytest.raises(ValueError, match="one row per sequence"):   # others are checked as ever
            c.decode(q[:1], two)


def test_parameters_are_taken_where_autograd_is_off():
    """A model's norm gains are parameters; without a graph to record, nothing is lost."""
    import torch
    c = _host_cache()
    gain = torch.nn.Parameter(torch.ones(64).bfloat16())
    q, two = torch.nn.Parameter(torch.ones(2, 4, 64).bfloat16()), torch.zeros(2, dtype=torch.int32)
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            assert c._gain(gain, "q_norm") == gain.data_ptr() and c._rows(q, "q", 4) == (2, 256)
            with pytest.raises(ValueError):   # never written to
                c.decode(q, two, out=q)
    for f in (lambda: c._gain(gain, "q_norm"), lambda: c._rows(q, "q", 4), lambda: c.decode(q, two)):
        with pytest.raises(ValueError):
            f()


def test_numbers_that_32_bits_would_cut_are_refused():
    import torch
    c = _host_cache()
    q, k, two = torch.ones(2, 4, 64).bfloat16(), torch.ones(2, 2, 64).bfloat16(), torch.zeros(2, dtype=torch.int32)
    for pairs in ((2 ** 32 + 8,), (8, 2 ** 32), (-2 ** 32 + 8, 8, 8), (2 ** 31,)):
        with pytest.raises(ValueError, match="32 bits"):
            c.append(q, k, k, two, two, rope_pairs=pairs)
    with pytest.raises(ValueError):
        c._rows(k[:1].expand(2 ** 32 + 1, 2, 64), "k", 2)
    for at in range(1, 7):
        c = _host_cache()
        c._shape = tuple(2 ** 32 + x if i == at else x for i, x in enumerate(c._shape))
        with pytest.raises(ValueError, match="32 bits"):
            c._desc(4)


def test_check_of_64_bit_lists_cuts_no_number():
    import torch
    from paper_2608_10824_amd import gvc
    c, far = _host_cache(), 2 ** 32
    c.check(torch.tensor([48, 0]), torch.tensor([0, -1]), torch.tensor([47, far]))
    for args in ((torch.tensor([far + 5, 0]),), (torch.tensor([-far, 0]),), (None, torch.tensor([far]), torch.tensor([3])),
                 (None, torch.tensor([far - 1]), torch.tensor([3])), (None, torch.tensor([0]), torch.tensor([far + 3]))):
        with pytest.raises(gvc.GvcError):
            c.check(*args)


# ---- the oracle
def test_oracle_rotation_is_the_prompt_oracle_s():
    """One axis over the whole head: the same as the decoder oracle's rotation."""
    x = np.random.default_rng(0).standard_normal((3, 64))
    for pos in (0, 1, 276, 100000):
        want = rope_row(x, pos, 1e4)
        got = np.stack([op.rope_norm(r, [pos], (32,), 1e4) for r in x])
        assert np.abs(got - want).max() < 1e-9


def test_oracle_axes_and_partial_rotation():
    x = np.random.default_rng(1).standard_normal(64)
    # equal positions on every axis: the axes do not matter
    assert np.allclose(op.rope_norm(x, [9, 9, 9], (8, 12, 12), 1e4), op.rope_norm(x, [9], (32,), 1e4), atol=1e-14)
    y = op.rope_norm(x, [5, 0, 0], (4, 6, 6), 1e4)
    assert np.array_equal(y[32:], x[32:])                                       # past 2 n: untouched
    assert np.array_equal(y[4:16], x[4:16]) and np.array_equal(y[20:32], x[20:32])   # axes at position 0
    assert np.allclose(y[:4] ** 2 + y[16:20] ** 2, x[:4] ** 2 + x[16:20] ** 2)
    n = op.rope_norm(x, [0], (32,), 1e4, gain=np.ones(64), eps=0.0)
    assert abs(np.mean(n * n) - 1) < 1e-12


def test_oracle_attention_is_the_prompt_oracle_s():
    """Every slot in sight over shuffled pages: the decoder oracle's row."""
    r = np.random.default_rng(2)
    k, v = r.standard_normal((7, 2, 16, 64)), r.standard_normal((7, 2, 64, 16))
    table = np.array([[5, 2, 0]])
    ks = np.concatenate([k[t] for t in table[0]], axis=1).transpose(1, 0, 2)
    vs = np.concatenate([v[t] for t in table[0]], axis=2).transpose(2, 0, 1)
    q = r.standard_normal((2, 64))
    for last in (0, 15, 16, 40):
        got = op.attend_row(q, 0, last, k, v, table, 0.125)[0]
        assert np.abs(got - attend_row(q, last, ks, vs)).max() < 1e-12
    assert op.seen_slots(9, 3, 2) == [0, 1, 7, 8, 9] and op.seen_slots(2, 5, 0) == [0, 1, 2] and op.seen_slots(-1, 0, 4) == []
    assert not op.attend_row(q, 0, -1, k, v, table, 0.125)[0].any()
    assert not op.attend_row(q, 0, 5, k, v, np.array([[9, 2, 0]]), 0.125)[0].any()
