"""The quantised paged cache on the host: refusals of the C ABI and of the
wrapper (nothing is launched, so no GPU is needed), and pins of its oracle."""
import ctypes

import numpy as np
import pytest

from oracle import quant as oq

P = 1 << 12   # an aligned address that nothing reads: every call below is refused


def _desc(**kw):
    from paper_2608_10824_amd import gvc
    d = gvc.PagedDesc(gvc.BF16, 8, 2, 64, 16, 4, 2, 3)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _rope(pairs=(32, 0, 0), theta=1e4, eps=1e-5):
    from paper_2608_10824_amd import gvc
    return gvc.PagedRope((ctypes.c_int32 * 3)(*pairs), theta, eps, None, None, None, 0)


def _append(desc, rope=None, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(q=P, qs=512, k=P, ks=128, v=P, vs=128, row_seq=P, row_slot=P, n=5, kp=P, kc=P, vp=P, vc=P, table=P, o=P,
             os=512)
    a.update(kw)
    gvc.quant_append(desc, rope or _rope(), *a.values(), None)


def _decode(desc, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(scale=0.125, window=0, sinks=0, q=P, qs=512, lengths=P, kp=P, kc=P, vp=P, vc=P, table=P, o=P, os=512,
             work=None, size=0)
    a.update(kw)
    gvc.quant_decode(desc, *a.values(), None)


def _prefill(desc, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(scale=0.125, window=0, sinks=0, q=P, qs=512, last=P, begin=P, n=5, kp=P, kc=P, vp=P, vc=P, table=P, o=P,
             os=512, work=None, size=0)
    a.update(kw)
    gvc.quant_prefill(desc, *a.values(), None)


def _read(desc, **kw):
    from paper_2608_10824_amd import gvc
    a = dict(row_seq=P, row_slot=P, n=5, kp=P, kc=P, vp=P, vc=P, table=P, k=P, ks=128, v=P, vs=128)
    a.update(kw)
    gvc.quant_read(desc, *a.values(), None)


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
    for f in (_append, _decode, _prefill, _read):
        _refused(f, d)
    _refused(gvc.quant_workspace, d, False, 1)


@pytest.mark.parametrize("call", [_append, _decode, _prefill, _read])
@pytest.mark.parametrize("kw", [dict(kp=None), dict(vp=None), dict(kc=None), dict(vc=None), dict(table=None),
                                dict(kp=P + 8), dict(vp=P + 4), dict(kc=P + 8), dict(vc=P + 1)])
def test_bad_pages_refused(call, kw):
    _refused(call, _desc(), **kw)


@pytest.mark.parametrize("kw", [dict(q=None), dict(o=None), dict(k=None), dict(v=None), dict(row_seq=None),
                                dict(row_slot=None), dict(n=-1), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4),
                                dict(o=P + 8), dict(qs=516), dict(ks=120), dict(vs=(1 << 32) + 8), dict(os=0),
                                dict(n=1 << 30), dict(rope=_rope(theta=0.0)), dict(rope=_rope(pairs=(30, 0, 0))),
                                dict(rope=_rope(eps=-1.0))])
def test_bad_append_refused(kw):
    _refused(_append, _desc(), **kw)


@pytest.mark.parametrize("call", [_decode, _prefill])
@pytest.mark.parametrize("kw", [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=3e38),
                                dict(window=-1), dict(sinks=-1), dict(q=None), dict(o=None), dict(q=P + 8),
                                dict(o=P + 2), dict(qs=508), dict(os=448)])
def test_bad_attention_refused(call, kw):
    _refused(call, _desc(), **kw)


def test_bad_lists_refused():
    _refused(_decode, _desc(), lengths=None)
    _refused(_prefill, _desc(), last=None)
    _refused(_prefill, _desc(), begin=None)
    _refused(_prefill, _desc(), n=-1)
    _refused(_prefill, _desc(), n=1 << 27)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=1 << 27), dict(row_seq=None), dict(row_slot=None), dict(k=P + 8),
                                dict(v=P + 2), dict(ks=120), dict(vs=132), dict(vs=(1 << 32) + 8)])
def test_bad_read_refused(kw):
    _refused(_read, _desc(), **kw)


def test_nothing_to_do():
    _append(_desc(), n=0, q=None, o=None, k=None, v=None, row_seq=None)
    _prefill(_desc(), n=0, q=None, o=None, last=None, begin=None)
    _read(_desc(), n=0, row_seq=None, k=None, v=None, kp=None)
    _read(_desc(), k=None, v=None)


def test_short_workspace_refused():
    from paper_2608_10824_amd import gvc
    d = _desc(max_pages=1000)
    need = gvc.quant_workspace(d, False, 2)
    assert need > 0
    _refused(_decode, d, code=gvc.GVC_ENOMEM)
    _refused(_decode, d, work=P, size=need - 1, code=gvc.GVC_ENOMEM)
    _refused(_decode, d, work=P + 8, size=need, code=gvc.GVC_ENOMEM)
    _refused(_prefill, d, work=None, size=need, code=gvc.GVC_ENOMEM)
    _refused(gvc.quant_workspace, d, True, 1 << 28)
    _refused(gvc.quant_workspace, d, False, 1, -1, 0)


def test_largest_tables():
    """2^30 slots in a row of the table and 2^27 entries in all are the most."""
    from paper_2608_10824_amd import gvc
    assert gvc.quant_workspace(_desc(n_seqs=4096, max_pages=1 << 15), False, 4096) > 0
    assert gvc.quant_workspace(_desc(n_seqs=1, max_pages=1 << 26), False, 1) > 0
    _refused(gvc.quant_workspace, _desc(n_seqs=4096, max_pages=(1 << 15) + 1), False, 4096)


# ---- the wrapper
def _tensors():
    import torch
    u8 = torch.zeros
    k, v = (u8(s, dtype=torch.uint8).view(torch.float8_e4m3fn) for s in ((4, 2, 16, 64), (4, 2, 64, 16)))
    ks, vs = (u8((4, 2, 16), dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in range(2))
    return k, ks, v, vs, torch.zeros(2, 3, dtype=torch.int32)


def _host_cache():
    """A cache over host memory, which only __init__ refuses: what its calls check comes before the C call."""
    import torch
    from paper_2608_10824_amd.paged import QuantPagedCache
    c = QuantPagedCache.__new__(QuantPagedCache)
    k, c.k_scales, v, c.v_scales, table = _tensors()
    c._hold(k, v, table, torch.bfloat16, -1, True)
    return c


def test_cache_refuses_other_tensors():
    import torch
    from paper_2608_10824_amd.paged import QuantPagedCache
    k, ks, v, vs, table = _tensors()
    for a in ((k, ks, v, vs, table), (k.view(torch.uint8), ks, v, vs, table), (k, ks.view(torch.uint8), v, vs, table),
              (k, ks, v.view(torch.float8_e5m2), vs, table), (k, ks, k, vs, table), (k[0], ks, v, vs, table),
              (k, ks[:3], v, vs, table), (k, ks, v, vs[..., :8], table), (k, ks, v, vs, table.long()),
              (k, ks, v, vs, table[0])):
        with pytest.raises(ValueError):
            QuantPagedCache(*a)
    with pytest.raises(ValueError, match="dtype"):
        QuantPagedCache(k, ks, v, vs, table, dtype=torch.float32)


def test_calls_refuse_other_tensors():
    import torch
    c = _host_cache()
    q, k, two = torch.ones(2, 4, 64).bfloat16(), torch.ones(2, 2, 64).bfloat16(), torch.zeros(2, dtype=torch.int32)
    for f in (lambda: c.read(two.long(), two), lambda: c.read(two, two[:1]), lambda: c.read(two[:, None], two),
              lambda: c.read(two, two, k_out=k.half()), lambda: c.read(two, two, v_out=k[:1]),
              lambda: c.read(two, two, k_out=q), lambda: c.read(two, two, k_out=k.clone().requires_grad_()),
              lambda: c.read(two, two, v_out=k.transpose(1, 2)), lambda: c.decode(q.half(), two),
              lambda: c.append(q, k.float(), k, two, two), lambda: c.prefill(q, two, two),
              lambda: c.decode(q.clone().requires_grad_(), two)):
        with pytest.raises(ValueError):
            f()


def test_forward_mode_duals_are_refused():
    import torch
    from torch.autograd import forward_ad
    c = _host_cache()
    q, k, two = torch.ones(2, 4, 64).bfloat16(), torch.ones(2, 2, 64).bfloat16(), torch.zeros(2, dtype=torch.int32)
    with forward_ad.dual_level():
        dk = forward_ad.make_dual(k, k.clone())
        for f in (lambda: c.read(two, two, k_out=dk), lambda: c.read(two, two, v_out=dk),
                  lambda: c.append(q, dk, k, two, two)):
            with pytest.raises(ValueError, match="tangent"):
                f()


def test_tables_and_lists_are_checked_as_for_16_bits():
    import torch
    from paper_2608_10824_amd import gvc
    c = _host_cache()
    c.page_table.copy_(torch.tensor([[3, 0, -1], [1, 7, 2]]))
    c.check(torch.tensor([32, 16]), torch.tensor([0, -1]), torch.tensor([31, 99]))
    with pytest.raises(gvc.GvcError, match="sequence 1"):
        c.check(torch.tensor([0, 17]))


# ---- the oracle
def test_oracle_codes():
    """Every code is its own rounding; half-way values go to the even code."""
    for c in list(range(127)) + list(range(128, 255)):
        got, scale = oq.quantise(np.array([448.0, oq.E4M3[c]]), "bf16")
        assert scale == 127 and oq.E4M3[got[1]] == oq.E4M3[c]
    for c in range(126):
        mid = (oq.E4M3[c] + oq.E4M3[c + 1]) / 2
        for x, want in ((mid, c + c % 2), (mid * (1 - 1e-12), c), (mid * (1 + 1e-12), c + 1)):
            assert oq.quantise(np.array([448.0, x]), "bf16")[0][1] == want
    assert oq.E4M3[0x08] == 2.0 ** -6 and oq.E4M3[0x38] == 1 and oq.E4M3[0x7e] == 448 and oq.E4M3[0x81] == -2.0 ** -9


def test_oracle_is_torch_s_rounding():
    import torch
    x = np.random.default_rng(0).standard_normal(4096).astype(np.float32) * 60
    x = np.concatenate([np.clip(x, -448, 448), [448.0]])
    codes, scale = oq.quantise(x, "bf16")
    assert scale == 127
    assert np.array_equal(codes, torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_oracle_scales():
    for size, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (224.1, 0), (1.0, -8), (0.875, -9), (1e-45, -126), (0.0, -126)):
        assert oq.scale_code(np.array([0.0, -size])) == e + 127
    assert oq.scale_code(np.array([np.nan, 1.0, np.inf])) == 127 - 8
    codes, s = oq.quantise(np.array([np.nan, 1.0, -np.inf]), "fp16")
    assert (codes[0] & 127, codes[1], codes[2]) == (127, 0x78, 255)
    # past the largest code of the type
    codes, s = oq.quantise(np.array([65504.0, -65000.0, 1e6]), "fp16")
    assert (oq.values(codes, np.array(s), "fp16") == [61440, -61440, 61440]).all()
    codes, s = oq.quantise(np.array([3.38e38, -3.2e38, 1.0]), "bf16")
    assert (oq.values(codes, np.array(s), "bf16") == [1.875 * 2.0 ** 127, -1.875 * 2.0 ** 127, 0]).all()


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_oracle_values_are_kept_when_quantised_again(t):
    r = np.random.default_rng(1)
    for _ in range(50):
        x = r.standard_normal(64) * 2.0 ** r.integers(-20, 10)
        once = oq.values(*[np.asarray(y) for y in oq.quantise(x, t)], t)
        again = oq.values(*[np.asarray(y) for y in oq.quantise(once, t)], t)
        assert np.array_equal(once, again)
        assert (np.abs(once - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * np.abs(x).max() / 224 + 2.0 ** -25).all()


def test_oracle_of_many_heads_is_that_of_one():
    x = np.random.default_rng(2).standard_normal((40, 64)) * 2.0 ** np.arange(-20, 20)[:, None]
    x[3] = 0
    x[4, 0] = 448
    x[5, 1], x[5, 2] = np.nan, np.inf
    for t in ("bf16", "fp16"):
        codes, scales = oq.quantise_heads(x, t)
        for i in range(40):
            c, s = oq.quantise(x[i], t)
            assert np.array_equal(c, codes[i]) and s == scales[i]
