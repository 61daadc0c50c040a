"""Refusals of the 8-bit block's entry points, their size queries and the oracle's own pins: no GPU needed."""
import ctypes as C

import numpy as np
import pytest

from oracle import block8 as ob
from paper_2602_07899_amd import tlq

FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)     # never dereferenced: validation fails first
BAD2 = C.c_void_p(0x1002)


def test_row_codes_refusals():
    l, p = tlq.lib(), tlq.params()

    def call(X=FAKE, n=4, c=72, ldx=72, f=FAKE, bits=8, par=p, codes=FAKE, ldc=128, steps=FAKE):
        return l.tlq_row_codes(X, n, c, ldx, f, bits, None if par is None else C.byref(par), codes, ldc, steps, None)
    for k in ("X", "codes", "steps", "par"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    assert call(bits=1) == call(bits=9) == call(bits=0) == tlq.ERR_UNSUPPORTED
    assert call(n=0) == call(c=0) == call(c=76, ldx=80) == call(ldx=64) == call(ldc=112) == call(n=1 << 31) == tlq.ERR_SHAPE
    assert call(ldc=1 << 31) == tlq.ERR_SHAPE
    assert call(X=ODD) == call(codes=ODD) == call(f=ODD) == call(ldx=76) == call(ldc=136) == call(steps=BAD2) == tlq.ERR_ALIGN


def test_linear_refusals():
    l, p = tlq.lib(), tlq.params(act_bits=8)

    def call(X=FAKE, n=4, ci=72, ldx=72, f=None, w=FAKE, co=5, ldw=128, ws=FAKE, par=p, Y=FAKE, ldy=8, work=FAKE, size=1 << 30):
        return l.tlq_linear_i8(X, n, ci, ldx, f, w, co, ldw, ws, C.byref(par), Y, ldy, work, size, None)
    for k in ("X", "w", "ws", "Y"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    assert call(par=tlq.params()) == call(ci=65544, ldx=65544, ldw=65664) == tlq.ERR_UNSUPPORTED
    assert call(n=0) == call(co=0) == call(ci=76, ldx=80) == call(ldw=112) == call(ldw=1 << 22) == call(co=1 << 29, ldy=1 << 29) == call(ldy=4) == call(ldx=64) == tlq.ERR_SHAPE
    assert call(X=ODD) == call(w=ODD) == call(ws=ODD) == call(f=ODD) == call(Y=ODD) == call(ldw=136) == call(ldy=12) == tlq.ERR_ALIGN
    assert call(work=None) == call(size=16) == tlq.ERR_WORKSPACE
    assert call(work=ODD) == tlq.ERR_ALIGN
    q = tlq.linear_i8_workspace_bytes
    assert q(0, 8) == q(4, 0) == q(4, 65544) == q(1 << 31, 8) == 0 and q(300, 72) == 300 * 128 + 1280
    # sums of parts of the codes: room for up to 64 tokens' at a time, up to 256 tokens
    assert q(3, 72) == 512 + 256 + 3 * 131072 and q(256, 128) == 256 * 128 + 1024 + 64 * 131072


def test_rope_refusals():
    l, p = tlq.lib(), tlq.params()

    def call(Q=FAKE, ldq=256, h=2, K=FAKE, ldk=128, kv=1, n=4, dh=128, rot=128, pairs=0, norm=1, eps=1e-6, wq=FAKE, wk=FAKE,
             pos=FAKE, inv=FAKE, qo=FAKE, ldqo=256, ko=FAKE, ldko=128):
        return l.tlq_qk_norm_rope(Q, ldq, h, K, ldk, kv, n, dh, rot, pairs, norm, eps, wq, wk, pos, inv, C.byref(p), qo, ldqo, ko, ldko, None)
    for k in ("Q", "K", "pos", "inv", "qo", "ko"):
        assert call(**{k: None}) == tlq.ERR_NULL, k
    for bad in (dict(dh=96), dict(dh=512), dict(pairs=2), dict(norm=2), dict(norm=0), dict(norm=0, wq=None), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf"))):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(n=0), dict(n=1 << 31), dict(n=1 << 26), dict(h=0), dict(kv=0), dict(h=65536, ldq=1 << 24, ldqo=1 << 24), dict(rot=-16), dict(rot=144),
                dict(rot=24), dict(ldq=248), dict(ldk=120), dict(ldqo=128), dict(ldko=64)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(Q=ODD), dict(K=ODD), dict(qo=ODD), dict(ko=ODD), dict(ldq=260), dict(ldko=132), dict(wq=ODD), dict(wk=ODD),
                dict(pos=BAD2), dict(inv=ODD)):
        assert call(**bad) == tlq.ERR_ALIGN, bad


def test_rows_beyond_the_threads_of_a_launch_are_refused():
    """A launch has fewer than 2^32 threads: rows of codes go eight to a block of up to eight waves, tokens' heads four tokens to
    a block of four."""
    l, p, a = tlq.lib(), tlq.params(), tlq.params(act_bits=8)
    for n, c in (((1 << 29) - 7, 8), ((1 << 29) - 7, 512), ((1 << 28) - 7, 520), ((1 << 26) - 7, 4096), ((1 << 26) - 7, 65536)):
        assert l.tlq_row_codes(FAKE, n, c, c, None, 8, C.byref(p), FAKE, -(-c // 128) * 128, FAKE, None) == tlq.ERR_SHAPE, (n, c)
        assert l.tlq_linear_i8(FAKE, n, c, c, None, FAKE, 8, -(-c // 128) * 128, FAKE, C.byref(a), FAKE, 8, FAKE, 1 << 60, None) == tlq.ERR_SHAPE
        assert tlq.linear_i8_workspace_bytes(n, c) == 0 < tlq.linear_i8_workspace_bytes(n - 1, c)
        # one row less is none of these (an address that is out of line is found behind the sizes)
        assert l.tlq_row_codes(ODD, n - 1, c, c, None, 8, C.byref(p), FAKE, -(-c // 128) * 128, FAKE, None) == tlq.ERR_ALIGN
    rope = lambda Q, n: l.tlq_qk_norm_rope(Q, 64, 1, FAKE, 64, 1, n, 64, 64, 0, 1, 1e-6, None, None, FAKE, FAKE, C.byref(p), FAKE, 64, FAKE, 64, None)
    assert rope(FAKE, (1 << 26) - 3) == rope(FAKE, (1 << 26) - 1) == tlq.ERR_SHAPE and rope(ODD, (1 << 26) - 4) == tlq.ERR_ALIGN


def _kv(**k):
    c = tlq.KvCache(C.sizeof(tlq.KvCache), 2, 128, 64, 10, 0x1000, 0x1000, 0x1000, 0x1000)
    b = tlq.KvBatch(C.sizeof(tlq.KvBatch), 3, 0x1000, 0x1000, 0x1000, 4, 4, 2, 200, 0)
    for name, v in k.items():
        setattr(c if name in dict(tlq.KvCache._fields_) and name != "struct_size" else b, name, v)
    return b, c


SHAPES = [dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(n_pages=0), dict(n_pages=1 << 31), dict(n_seq=0), dict(n_seq=65536),
          dict(max_pages=0), dict(ld_table=3), dict(max_new=0), dict(max_len=1), dict(max_len=(1 << 30) + 1)]
UNSUPPORTED = [dict(head_dim=96), dict(head_dim=256), dict(page=8), dict(page=48), dict(page=512), dict(reserved=1)]


def test_cache_refusals():
    l, p = tlq.lib(), tlq.params()

    def append(K=FAKE, ldk=256, V=FAKE, ldv=256, n=6, par=p, size_b=None, size_c=None, **k):
        b, c = _kv(**k)
        b.struct_size, c.struct_size = size_b or b.struct_size, size_c or c.struct_size
        return l.tlq_kv_append(K, ldk, V, ldv, n, C.byref(b), C.byref(c), None if par is None else C.byref(par), None)

    def attend(Q=FAKE, ldq=512, n=6, heads=4, scale=0.0, Out=FAKE, ldo=512, work=FAKE, size=1 << 40, size_b=None, size_c=None, **k):
        b, c = _kv(**k)
        b.struct_size, c.struct_size = size_b or b.struct_size, size_c or c.struct_size
        return l.tlq_kv_attention(Q, ldq, n, heads, scale, C.byref(b), C.byref(c), C.byref(p), Out, ldo, work, size, None)
    for call in (append, attend):
        for bad in SHAPES:
            assert call(**bad) == tlq.ERR_SHAPE, bad
        for bad in UNSUPPORTED + [dict(size_b=48), dict(size_c=48)]:
            assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
        for name in ("cu_new", "lens", "table", "k", "k_step", "v", "v_step"):
            assert call(**{name: None}) == tlq.ERR_NULL, name
            assert call(**{name: 0x1002}) == tlq.ERR_ALIGN, name
        assert call(k=0x1008) == call(v=0x1008) == tlq.ERR_ALIGN
        assert call(n=0) == call(n=1 << 31) == tlq.ERR_SHAPE
    assert append(K=None) == append(V=None) == append(par=None) == tlq.ERR_NULL
    assert append(ldk=248) == append(ldv=128) == tlq.ERR_SHAPE
    assert append(K=ODD) == append(V=ODD) == append(ldk=260) == append(ldv=260) == tlq.ERR_ALIGN
    assert attend(Q=None) == attend(Out=None) == tlq.ERR_NULL
    assert attend(heads=3) == attend(heads=0) == attend(ldq=504) == attend(ldo=256) == attend(heads=65536) == tlq.ERR_SHAPE
    # more blocks than a launch can have
    assert append(n=1 << 30, n_seq=1000, max_new=1 << 20, max_len=1 << 20, page=16) == tlq.ERR_SHAPE
    assert attend(n=1 << 28, heads=4, max_new=1 << 28, max_len=1 << 28, n_kv_heads=4, ldq=512) == tlq.ERR_SHAPE
    assert attend(n=1 << 21, heads=2, max_new=1 << 21, max_len=1 << 21, n_seq=65535, n_kv_heads=2, ldq=256, ldo=256) == tlq.ERR_SHAPE
    assert attend(scale=float("nan")) == attend(scale=float("inf")) == tlq.ERR_UNSUPPORTED
    assert attend(Q=ODD) == attend(Out=ODD) == attend(ldq=516) == attend(ldo=516) == tlq.ERR_ALIGN
    long = dict(max_len=100000, max_pages=2000, ld_table=2000, n=3)
    assert attend(work=None, **long) == attend(size=64, **long) == tlq.ERR_WORKSPACE
    assert attend(work=ODD, **long) == tlq.ERR_ALIGN


def test_cache_size_query():
    q = lambda n, heads, **k: tlq.kv_attention_workspace_bytes(n, heads, *_kv(**k))
    for bad in SHAPES + UNSUPPORTED:
        assert q(6, 4, **bad) == 0
    assert q(0, 4) == q(6, 3) == 0
    none = dict(cu_new=None, lens=None, table=None, k=None, v=None, k_step=None, v_step=None)
    long = dict(max_len=100000, max_pages=2000, ld_table=2000)
    assert q(3, 4, **long) > 3 * 4 * 128 * 4 and q(3, 4, **long) == q(3, 4, **long, **none)       # sizes only
    # the table's room bounds the keys
    assert q(3, 4, max_len=1 << 30) == q(3, 4, max_len=256)


def test_binding_refusals():
    """Tensors of another type, shape or device than the call reads are refused before the library is called."""
    import torch
    p = tlq.params(act_bits=8)
    x, w, s = torch.zeros((2, 128), dtype=torch.float16), torch.zeros((3, 128), dtype=torch.int8), torch.zeros(3)
    y = torch.zeros((2, 8), dtype=torch.float16)[:, :3]
    for bad in (lambda: tlq.linear_i8(x, w, s, p, y),                              # not on a GPU
                lambda: tlq.linear_i8(x.float(), w, s, p, y),
                lambda: tlq.row_codes(x, 8, p, w[:2].float(), s[:2]),
                lambda: tlq.qk_norm_rope(x, x, 128, torch.zeros(2), None, p, x, x)):
        with pytest.raises(ValueError):
            bad()
    k = torch.zeros((4, 2, 16, 64), dtype=torch.int8)
    v, st = torch.zeros((4, 2, 64, 16), dtype=torch.int8), torch.zeros((4, 2))
    c = tlq.kv_cache(k, st, v, st.clone())
    assert (c.n_pages, c.n_kv_heads, c.page, c.head_dim) == (4, 2, 16, 64)
    for bad in (lambda: tlq.kv_cache(k, st, k, st), lambda: tlq.kv_cache(k, st[:3], v, st), lambda: tlq.kv_cache(k[:, :1], st[:, :1], v[:, :1], st[:, :1])):
        with pytest.raises(ValueError):
            bad()
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    b = tlq.kv_batch(i(3), i(2), i(2, 5), 1, 40)
    assert (b.n_seq, b.max_pages, b.ld_table) == (2, 5, 5)
    assert tlq.kv_batch(i(3), i(2), i(2, 9)[:, :5], 1, 40).ld_table == 9
    for bad in (lambda: tlq.kv_batch(i(2), i(2), i(2, 5), 1, 40), lambda: tlq.kv_batch(i(3), i(2), i(3, 5), 1, 40),
                lambda: tlq.kv_batch(i(3), i(2), i(5, 2).t(), 1, 40), lambda: tlq.kv_append(x, x, b, c, p),
                lambda: tlq.kv_attention(x, 2, b, c, p, x)):
        with pytest.raises(ValueError):
            bad()


def test_tables_whose_rows_overlap_are_refused():
    """Rows that lie on each other (an expanded table) would be read a row's length apart, behind the table's end."""
    import torch
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    for table in (i(1, 5).expand(2, 5), torch.as_strided(i(9), (2, 5), (4, 1)), i(1, 1).expand(2, 1)):
        with pytest.raises(ValueError):
            tlq.kv_batch(i(3), i(2), table, 1, 40)
    b = tlq.kv_batch(i(2), i(1), torch.as_strided(i(9), (1, 5), (0, 1)), 1, 40)      # (of a single row the stride is never used)
    assert b.max_pages == 5 <= b.ld_table
    assert tlq.kv_batch(i(3), i(2), i(2, 1), 1, 16).ld_table == 1


def test_bounds_beyond_32_bits_are_refused():
    """A bound of tokens that the structure cannot hold is not cut to its low bits."""
    import torch
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    for new, most in ((1, (1 << 32) + 40), ((1 << 32) + 1, 40), (1, 1 << 31), (1 - (1 << 32), 40), (1, 40 - (1 << 32))):
        with pytest.raises(ValueError):
            tlq.kv_batch(i(3), i(2), i(2, 5), new, most)
    assert tlq.kv_batch(i(3), i(2), i(2, 5), 1, (1 << 31) - 1).max_len == (1 << 31) - 1      # (the call refuses it)


# ------------------------------------------------------------------ pins of the oracle
def test_oracle_attention_by_hand():
    """One key head, two tokens, weights 1 / 3 and 2 / 3 by hand; the first row sees itself only."""
    kc, vc = np.zeros((1, 1, 16, 64), np.int8), np.zeros((1, 1, 64, 16), np.int8)
    kc[0, 0, 1, 0] = 2
    vc[0, 0, 0, :2], vc[0, 0, 1, :2] = [3, 6], [9, 0]
    ks, vs = np.full((1, 1), np.log(2.0) / 2, np.float32), np.full((1, 1), 0.5, np.float32)
    q = np.zeros((2, 64))
    q[:, 0] = 1.0
    out, mag, _ = ob.kv_attention(q, 1, kc, ks, vc, vs, [0, 2], [2], np.zeros((1, 1), int), 16, scale=1.0)
    np.testing.assert_allclose(out[:, :2], [[1.5, 4.5], [2.5, 1.5]], rtol=1e-6)
    np.testing.assert_allclose(mag[:, :2], [[1.5, 4.5], [2.5, 1.5]], rtol=1e-6)


def test_oracle_append_by_hand():
    """A page with one token of step 1 meets a token of twice its size: its codes are halved, ties to even."""
    codes, steps = np.zeros((1, 1, 16, 64), np.int8), np.ones((1, 1), np.float32)
    codes[0, 0, 0, :4] = [127, 3, 1, -5]
    x = np.zeros((1, 64), np.float32)
    x[0, :3] = [254.0, -2.0, 1.0]
    ob.kv_append(x, codes, steps, [0, 1], [2], np.zeros((1, 1), int), 16, False)
    assert steps[0, 0] == 2.0
    assert codes[0, 0, 0, :4].tolist() == [64, 2, 0, -2] and codes[0, 0, 1, :3].tolist() == [127, -1, 0]


def test_oracle_rotation_keeps_lengths_and_products():
    """A rotation keeps a head's length, and products of two rotated heads depend on the distance of their positions only."""
    g = np.random.default_rng(1)
    x = g.standard_normal((4, 64))
    inv = 100.0 ** (-np.arange(32) / 32)
    for pairs in (False, True):
        r = lambda v, p: ob.qk_norm_rope(v[None], 64, np.array([p]), inv, norm=False, interleaved=pairs)[0]
        np.testing.assert_allclose(np.linalg.norm(r(x[0], 17)), np.linalg.norm(x[0]), rtol=1e-12)
        np.testing.assert_allclose(r(x[0], 17) @ r(x[1], 11), r(x[0], 106) @ r(x[1], 100), rtol=1e-9)
    u = ob.qk_norm_rope(x, 64, np.zeros(4, int), inv, eps=0.0)
    np.testing.assert_allclose((u ** 2).mean(axis=1), 1.0, rtol=1e-12)


def test_oracle_linear_is_exact_on_its_grid():
    x = np.arange(-127, 128, dtype=np.float32)[None, :].repeat(2, 0)
    x[1] *= 4
    codes, steps = ob.row_codes(x, 8)
    assert np.array_equal(codes[0], x[0]) and np.array_equal(codes[1], x[0]) and steps.tolist() == [1.0, 4.0]
    w = np.full((1, 255), 3, np.int8)
    w[0, :127] = 0
    assert ob.linear_i8(x, 8, w, np.array([0.5], np.float32)).tolist() == [[8128 * 1.5], [8128 * 6.0]]
