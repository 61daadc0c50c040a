"""Refusals of the block's other low-bit entry points, their size queries and the oracle's own pins: no GPU needed."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import block8 as ob
from oracle import lowbit as lo
from paper_2602_07899_amd import tlq

FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)     # never dereferenced: validation fails first
BAD2 = C.c_void_p(0x1002)


def test_add_norm_codes_refusals():
    l, p = tlq.lib(), tlq.params()

    def call(H=FAKE, ldh=72, Z=FAKE, ldz=72, n=4, c=72, w=FAKE, eps=1e-6, bits=8, par=p, out=FAKE, ldo=72, codes=FAKE, ldc=128, steps=FAKE):
        return l.tlq_add_norm_codes(H, ldh, Z, ldz, n, c, w, eps, bits, None if par is None else C.byref(par), out, ldo, codes, ldc, steps, None)
    for k in ("H", "codes", "steps", "par"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    for bad in (dict(bits=1), dict(bits=9), dict(bits=0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(c=65544, ldh=65544, ldz=65544, ldo=65544, ldc=65664)):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(n=0), dict(n=(1 << 21) + 1), dict(c=0), dict(c=76, ldh=80, ldz=80, ldo=80), dict(ldh=64), dict(ldz=64), dict(ldo=64), dict(ldc=112), dict(ldc=1 << 31)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(H=ODD), dict(Z=ODD), dict(out=ODD), dict(codes=ODD), dict(w=ODD), dict(steps=BAD2), dict(ldh=76), dict(ldz=76), dict(ldo=76), dict(ldc=136)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    # what is not there has no stride (an address that is out of line is found behind the sizes)
    assert call(Z=None, ldz=0, out=None, ldo=0, w=None, steps=BAD2) == tlq.ERR_ALIGN and call(n=1 << 21, H=ODD) == tlq.ERR_ALIGN


def test_linear_codes_refusals():
    l, p = tlq.lib(), tlq.params()

    def call(x=FAKE, ldx=128, st=FAKE, n=4, ci=72, w=FAKE, co=5, ldw=128, ws=FAKE, bias=FAKE, act=1, R=FAKE, ldr=8, mul=1, par=p, Y=FAKE, ldy=8,
             work=FAKE, size=1 << 30):
        return l.tlq_linear_codes(x, ldx, st, n, ci, w, co, ldw, ws, bias, act, R, ldr, mul, None if par is None else C.byref(par), Y, ldy, work, size, None)
    for k in ("x", "st", "w", "ws", "par", "Y"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    for bad in (dict(act=-1), dict(act=4), dict(mul=2), dict(mul=-1), dict(R=None), dict(ci=65544, ldx=65664, ldw=65664)):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(n=0), dict(n=1 << 31), dict(co=0), dict(ci=76), dict(ci=136), dict(ldx=112), dict(ldx=1 << 22), dict(ldw=112), dict(ldw=1 << 22),
                dict(co=1 << 29, ldy=1 << 29, ldr=1 << 29), dict(ldy=4), dict(ldr=4), dict(ldr=0)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(x=ODD), dict(st=BAD2), dict(w=ODD), dict(ws=ODD), dict(bias=ODD), dict(R=ODD), dict(Y=ODD), dict(ldx=136), dict(ldw=136), dict(ldy=12), dict(ldr=12)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    f = tlq.params(yref_dtype=tlq.F32)
    assert call(par=f, ldy=6) == call(par=f, ldr=6) == tlq.ERR_ALIGN and call(par=f, ldy=12, ldr=12, work=None) == tlq.ERR_WORKSPACE
    assert call(work=None) == call(size=16) == tlq.ERR_WORKSPACE and call(work=ODD) == tlq.ERR_ALIGN
    q = tlq.linear_codes_workspace_bytes
    assert q(0, 8) == q(4, 0) == q(4, 65544) == q(1 << 31, 8) == q(257, 72) == 0 and q(3, 72) == 3 * 131072 and q(256, 128) == 64 * 131072


def test_rope_axes_refusals():
    l, p = tlq.lib(), tlq.params()

    def call(Q=FAKE, ldq=256, h=2, K=FAKE, ldk=128, kv=1, n=4, dh=128, rot=128, pairs=0, norm=1, eps=1e-6, wq=FAKE, wk=FAKE,
             pos=FAKE, ldp=4, axes=3, axis=FAKE, inv=FAKE, qo=FAKE, ldqo=256, ko=FAKE, ldko=128):
        return l.tlq_qk_norm_rope_axes(Q, ldq, h, K, ldk, kv, n, dh, rot, pairs, norm, eps, wq, wk, pos, ldp, axes, axis, inv, C.byref(p), qo, ldqo, ko,
                                       ldko, None)
    for k in ("Q", "K", "pos", "axis", "inv", "qo", "ko"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    for bad in (dict(axes=0), dict(axes=5), dict(axes=-1), dict(dh=96), dict(pairs=2), dict(norm=0), dict(eps=-1.0)):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(ldp=3), dict(ldp=1 << 40), dict(n=0), dict(n=1 << 26, ldp=1 << 26), dict(rot=24), dict(ldq=248), dict(ldko=64)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(axis=BAD2), dict(pos=BAD2), dict(inv=ODD), dict(Q=ODD), dict(ldko=132), dict(wk=ODD)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    assert call(rot=0, axis=None, inv=None, Q=ODD) == tlq.ERR_ALIGN


def _kv(**k):
    c = tlq.Kv4Cache(C.sizeof(tlq.Kv4Cache), 2, 128, 64, 10, 0x1000, 0x1000, 0x1000, 0x1000)
    b = tlq.KvBatch(C.sizeof(tlq.KvBatch), 3, 0x1000, 0x1000, 0x1000, 4, 4, 2, 200, 0)
    for name, v in k.items():
        setattr(c if name in dict(tlq.Kv4Cache._fields_) and name != "struct_size" else b, name, v)
    return b, c


SHAPES = [dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(n_pages=0), dict(n_pages=1 << 31), dict(n_seq=0), dict(n_seq=65536),
          dict(max_pages=0), dict(ld_table=3), dict(max_new=0), dict(max_len=1), dict(max_len=(1 << 30) + 1)]
UNSUPPORTED = [dict(head_dim=96), dict(head_dim=256), dict(page=8), dict(page=48), dict(page=512), dict(reserved=1)]


def test_cache_refusals():
    l, p = tlq.lib(), tlq.params()

    def made(size_b, size_c, k):
        b, c = _kv(**k)
        b.struct_size, c.struct_size = size_b or b.struct_size, size_c or c.struct_size
        return C.byref(b), C.byref(c)

    def append(K=FAKE, ldk=256, V=FAKE, ldv=256, n=6, par=p, size_b=None, size_c=None, **k):
        b, c = made(size_b, size_c, k)
        return l.tlq_kv4_append(K, ldk, V, ldv, n, b, c, None if par is None else C.byref(par), None)

    def read(K=FAKE, ldk=256, V=FAKE, ldv=256, n=6, par=p, size_b=None, size_c=None, **k):
        b, c = made(size_b, size_c, k)
        return l.tlq_kv4_read(b, c, None if par is None else C.byref(par), n, K, ldk, V, ldv, None)

    def attend(Q=FAKE, ldq=512, n=6, heads=4, scale=0.0, Out=FAKE, ldo=512, work=FAKE, size=1 << 40, size_b=None, size_c=None, **k):
        b, c = made(size_b, size_c, k)
        return l.tlq_kv4_attention(Q, ldq, n, heads, scale, b, c, C.byref(p), Out, ldo, work, size, None)
    for call in (append, read, attend):
        for bad in SHAPES:
            assert call(**bad) == tlq.ERR_SHAPE, bad
        for bad in UNSUPPORTED + [dict(size_b=48), dict(size_c=48)]:
            assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
        for name in ("cu_new", "lens", "table", "k", "k_step", "v", "v_step"):
            assert call(**{name: None}) == tlq.ERR_NULL, name
            assert call(**{name: 0x1002}) == tlq.ERR_ALIGN, name
        for name in ("k", "v", "k_step", "v_step"):
            assert call(**{name: 0x1008}) == tlq.ERR_ALIGN, name
        assert call(n=0) == call(n=1 << 31) == tlq.ERR_SHAPE
    for call in (append, read):
        assert call(K=None, V=None) == call(par=None) == tlq.ERR_NULL
        assert call(ldk=248) == call(ldv=128) == tlq.ERR_SHAPE
        assert call(K=ODD) == call(V=ODD) == call(ldk=260) == call(ldv=260) == tlq.ERR_ALIGN
        # more threads than a launch can have, and the last that fits (found behind: the address)
        big = dict(n=1 << 20, n_seq=32767, max_new=4064, max_len=4064)       # 2 x ceil(509 / 4) / 4 = 64 blocks a sequence
        assert call(**{**big, "max_new": 4096 * 4, "max_len": 1 << 20, "n_seq": 65535}) == tlq.ERR_SHAPE
        assert call(K=ODD, **big) == tlq.ERR_ALIGN
        # one token of many heads: a wave each.  128 x 65535 blocks are fewer than 2^23, 129 are not
        one = dict(n=1 << 20, n_seq=65535, max_new=1, max_len=1, n_kv_heads=512, ldk=513 * 128, ldv=513 * 128)
        assert call(K=ODD, **one) == tlq.ERR_ALIGN
        assert call(**{**one, "n_kv_heads": 513}) == tlq.ERR_SHAPE
        # 57 tokens lie in eight eights at most, a wave's of 64 channels; 58 can lie in nine
        most = dict(n=1 << 20, n_seq=65535, max_new=57, max_len=58, n_kv_heads=512, head_dim=64, ldk=512 * 64, ldv=512 * 64)
        assert call(K=ODD, **most) == tlq.ERR_ALIGN
        assert call(**{**most, "max_new": 58}) == tlq.ERR_SHAPE
    assert append(K=None) == append(V=None) == tlq.ERR_NULL
    assert read(K=None, ldk=0, V=ODD) == read(V=None, ldv=0, K=ODD) == tlq.ERR_ALIGN
    assert attend(Q=None) == attend(Out=None) == tlq.ERR_NULL
    assert attend(heads=3) == attend(heads=0) == attend(ldq=504) == attend(ldo=256) == attend(heads=65536) == tlq.ERR_SHAPE
    assert attend(n=1 << 28, heads=4, max_new=1 << 28, max_len=1 << 28, n_kv_heads=4, ldq=512) == tlq.ERR_SHAPE
    assert attend(scale=float("nan")) == attend(scale=float("inf")) == tlq.ERR_UNSUPPORTED
    assert attend(Q=ODD) == attend(Out=ODD) == attend(ldq=516) == attend(ldo=516) == tlq.ERR_ALIGN
    long = dict(max_len=100000, max_pages=2000, ld_table=2000, n=3)
    assert attend(work=None, **long) == attend(size=64, **long) == tlq.ERR_WORKSPACE
    assert attend(work=ODD, **long) == tlq.ERR_ALIGN


def test_cache_size_query():
    q = lambda n, heads, **k: tlq.kv4_attention_workspace_bytes(n, heads, *_kv(**k))
    for bad in SHAPES + UNSUPPORTED:
        assert q(6, 4, **bad) == 0
    assert q(0, 4) == q(6, 3) == 0
    none = dict(cu_new=None, lens=None, table=None, k=None, v=None, k_step=None, v_step=None)
    long = dict(max_len=100000, max_pages=2000, ld_table=2000)
    assert q(3, 4, **long) > 3 * 4 * 128 * 4 and q(3, 4, **long) == q(3, 4, **long, **none)       # sizes only
    assert q(3, 4, max_len=1 << 30) == q(3, 4, max_len=256)                                      # the table's room bounds the keys


def test_binding_refusals():
    """Tensors of another type, shape or device than the call reads are refused before the library is called."""
    import torch
    p = tlq.params(act_bits=8)
    half = lambda *n: torch.zeros(n, dtype=torch.float16)
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    x, c8, s = half(2, 128), torch.zeros((2, 128), dtype=torch.int8), torch.zeros(2)
    k, v, ks, vs = i(4, 2, 16, 8), i(4, 2, 64, 2), half(4, 2, 16, 2), half(4, 2, 2, 16)
    c = tlq.kv4_cache(k, ks, v, vs)
    assert (c.n_pages, c.n_kv_heads, c.page, c.head_dim) == (4, 2, 16, 64)
    b = tlq.kv_batch(i(3), i(2), i(2, 5), 1, 40)
    other = tlq.kv_cache(torch.zeros((4, 2, 16, 64), dtype=torch.int8), torch.zeros((4, 2)), torch.zeros((4, 2, 64, 16), dtype=torch.int8), torch.zeros((4, 2)))
    for bad in (lambda: tlq.add_norm_codes(x, None, p, c8, s),                     # not on a GPU
                lambda: tlq.linear_codes(c8, s, 128, c8, s, p, half(2, 8)[:, :2]),
                lambda: tlq.qk_norm_rope_axes(x, x, 128, i(3, 2), i(64), torch.zeros(64, dtype=torch.float64), p, x, x),
                lambda: tlq.kv4_cache(k, ks, k, vs), lambda: tlq.kv4_cache(k, ks[:3], v, vs), lambda: tlq.kv4_cache(k, vs, v, ks),
                lambda: tlq.kv4_cache(k[:, :1], ks[:, :1], v[:, :1], vs[:, :1]), lambda: tlq.kv4_read(b, c, p),
                lambda: tlq.kv4_append(x, x, b, c, p), lambda: tlq.kv4_read(b, c, p, x, x), lambda: tlq.kv4_attention(x, 2, b, c, p, x),
                lambda: tlq.kv4_attention(x, 2, b, other, p, x), lambda: tlq.kv_attention(x, 2, b, c, p, x)):
        with pytest.raises(ValueError):
            bad()
    # a cache of the other kind is no argument of the library's function either
    for fn, cache in ((tlq.lib().tlq_kv4_append, other), (tlq.lib().tlq_kv_append, c)):
        with pytest.raises(C.ArgumentError):
            fn(FAKE, 128, FAKE, 128, 2, C.byref(b), C.byref(cache), C.byref(p), None)


# ------------------------------------------------------------------ pins of the oracle
def test_oracle_words_by_hand():
    """Element e lies in the four bits from 4 (e / 2) + 16 (e % 2) up."""
    c = np.array([[-8, -7, -6, -5, 0, 1, 6, 7]])
    # even elements -8 -6 0 6 -> 0 2 8 14 in the low half, odd ones -7 -5 1 7 -> 1 3 9 15 in the high half
    assert lo.pack(c).view(np.uint32).tolist() == [[0xF931E820]]
    g = np.random.default_rng(1).integers(-8, 8, (3, 5, 64))
    assert np.array_equal(lo.unpack(lo.pack(g)), g)


def test_oracle_quantiser_by_hand():
    x = np.zeros((1, 64), np.float32)
    x[0, :6] = [7.0, -3.5, 0.5, 1.5, np.nan, -np.inf]         # step 1; ties to even
    x[0, 32] = 1e-6                                           # below the floor
    c, s = lo.quantise(x)
    assert s.tolist() == [[1.0, float(np.float16(round(1e-5 / 7 * 2 ** 24) * 2.0 ** -24))]] and c[0, :6].tolist() == [7, -4, 0, 2, 0, -7] and c[0, 32] == 1
    big, sb = lo.quantise(np.full((1, 32), 3e38, np.float32))
    assert sb[0, 0] == 9344.0 and big[0, 0] == 7


def test_oracle_steps_keep_products_exact():
    """A step has eight significant bits, so that seven of them are a half."""
    m = np.exp(np.random.default_rng(2).uniform(math.log(1e-5), math.log(7e4), 4000)).astype(np.float32)
    x = np.zeros((4000, 32), np.float32)
    x[:, 0] = m
    _, s = lo.quantise(x)
    for k in range(1, 9):
        v = k * s.astype(np.float64)
        ok = v <= 65504
        assert np.array_equal(v[ok], v[ok].astype(np.float16).astype(np.float64)) and (k == 8 or ok.all())


def test_oracle_cache_by_hand():
    """Two tokens into a begun page and back; what is not new stays."""
    codes, steps = np.full((2, 1, 16, 32), 3, np.int8), np.full((2, 1, 16, 1), 2.0, np.float16)
    x = np.zeros((2, 32), np.float32)
    x[0, 0], x[1, 1] = 14.0, -0.875
    cu, lens, table = [0, 2], [17], np.array([[1, 0]])
    lo.kv4_append(x, codes, steps, cu, lens, table, 32, False)
    assert codes[1, 0, 15, :2].tolist() == [7, 0] and steps[1, 0, 15, 0] == 2.0 and codes[0, 0, 0, :2].tolist() == [0, -7] and steps[0, 0, 0, 0] == 0.125
    assert (codes[1, 0, :15] == 3).all() and (codes[0, 0, 1:] == 3).all()
    back = lo.kv4_read(codes, steps, cu, lens, table, 3, 32, False)
    assert back[0, 0] == 14.0 and back[1, 1] == -0.875 and np.isnan(back[2]).all()


def test_oracle_attention_is_that_of_the_other_cache():
    """On pools that both caches can hold."""
    g = np.random.default_rng(3)
    kc, vc = g.integers(-7, 8, (5, 2, 16, 64)).astype(np.int8), g.integers(-7, 8, (5, 2, 64, 16)).astype(np.int8)
    ks = vs = np.full((5, 2), 0.25, np.float32)
    q, table = g.standard_normal((6, 4 * 64)), np.array([[3, 0, 4], [-1, 2, 9]])
    args = ([0, 4, 6], [40, 30], table, 48)
    a = ob.kv_attention(q, 4, kc, ks, vc, vs, *args)
    st = np.full((5, 2, 16, 2), 0.25, np.float16)
    b = lo.attention(q, 4, lo.values(kc, st, False), lo.values(vc, st.transpose(0, 1, 3, 2), True), *args)
    for x, y in zip(a, b):
        np.testing.assert_allclose(x, y, rtol=1e-12, atol=1e-300)


def test_oracle_norm_by_hand():
    """Two channels of 3 and 4: a mean square of 12.5."""
    h = np.zeros((1, 8), np.float32)
    h[0, :2] = [3.0, 4.0]
    out, c, s = lo.add_norm_codes(h, h, None, 0.0, 8, False)
    assert out[0, :2].tolist() == [6.0, 8.0] and c[0, :2].tolist() == [95, 127]
    np.testing.assert_allclose(s, 8.0 / math.sqrt(100.0 / 8.0) / 127.0, rtol=1e-6)


def test_oracle_activations():
    for kind in (1, 2, 3):
        a = lo.act(np.array([-40.0, -3.0, 0.0, 3.0, 40.0]), kind)
        assert a[2] == 0.0 and abs(a[0]) < 1e-15 and abs(a[4] - 40.0) < 1e-12 and abs(a[3] - a[1] - 3.0) < 1e-12      # a(v) - a(-v) = v
    np.testing.assert_allclose(lo.act(1.0, 1), 0.7310585786300049, rtol=1e-14)
    np.testing.assert_allclose(lo.act(1.0, 3), 0.8413447460685429, rtol=1e-14)
    np.testing.assert_allclose(lo.act(1.0, 2), 0.5 * (1 + math.tanh(math.sqrt(2 / math.pi) * 1.044715)), rtol=1e-14)


def test_oracle_rotation_with_one_axis_is_the_other():
    g = np.random.default_rng(4)
    x, inv = g.standard_normal((4, 128)), 100.0 ** (-np.arange(32) / 32)
    pos = np.array([5, 0, -3, 70000])
    for pairs in (False, True):
        for axis in (np.zeros(32, int), np.arange(32) % 3):
            a = lo.norm_rope_axes(x, 64, np.stack([pos] * 3), axis, inv, interleaved=pairs)
            np.testing.assert_allclose(a, ob.qk_norm_rope(x, 64, pos, inv, interleaved=pairs), rtol=1e-10, atol=1e-12)
