"""A decoder block in 8 bits on the GPU against the 64-bit oracle: codes of rows, the integer linear, normalised and rotated
queries and keys, appends to the paged cache, attention over it, a run of them together, captured graphs, streams."""
import numpy as np
import pytest

from oracle import block8 as ob
from oracle import tlq_oracle as orc
from paper_2602_07899_amd import tlq

pytestmark = pytest.mark.gpu

HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step, relative
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}    # half of the smallest step
U = 2.0 ** -24
CODE = {"f16": tlq.F16, "bf16": tlq.BF16, "f32": tlq.F32}


def tt(dt):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dt]


def rnd(a, dt):
    """float32 values that dt holds exactly."""
    a = np.asarray(a, np.float32)
    return a.astype(np.float16).astype(np.float32) if dt == "f16" else np.asarray(orc.round_to_bf16(a), np.float32)


def dev(a, gpu, dt=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to(gpu)
    return t if dt is None else t.to(tt(dt))


def host(t):
    return t.detach().double().cpu().numpy()


def spread(a, gpu, dt, left=8, right=16):
    """A column slice of a wider matrix that holds `a`, and the matrix."""
    import torch
    wide = torch.full((a.shape[0], left + -(-a.shape[1] // 8) * 8 + right), 3.0, dtype=tt(dt), device=gpu)
    part = wide[:, left:left + a.shape[1]]
    part.copy_(dev(a, gpu, dt))
    return part, wide


def within(got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) / bound)), np.argwhere(bad)[:4].tolist())


# ------------------------------------------------------------------ row codes, integer linear
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,c,bits,scaled", [(1, 8, 8, True), (3, 72, 8, False), (17, 128, 4, True), (9, 1096, 2, True),
                                             (130, 520, 6, False), (2, 13824, 8, True), (3, 1032, 8, True),
                                             (5, 4104, 8, True), (2, 8200, 5, True), (3, 16392, 8, True), (70, 1024, 8, True)])
def test_row_codes_are_exact(gpu, dt, n, c, bits, scaled):
    import torch
    g = np.random.default_rng([21, n, c])
    x = rnd(g.standard_normal((n, c)) * np.exp(g.standard_normal((n, 1)) * 3), dt)
    x[0, :] = 0.0 if n > 1 else x[0, :]                       # a row of zeros: the floor
    f = np.exp(g.standard_normal(c)).astype(np.float32) if scaled else None
    p = tlq.params(x_dtype=CODE[dt])
    c8 = -(-c // 128) * 128
    wide = torch.full((n, c8 + 32), 77, dtype=torch.int8, device=gpu)
    steps = torch.empty(n, dtype=torch.float32, device=gpu)
    xt, _ = spread(x, gpu, dt)
    tlq.row_codes(xt, bits, p, wide[:, 16:16 + c8], steps, factor=None if f is None else dev(f, gpu))
    want, wsteps = ob.row_codes(x, bits, f)
    got = wide.cpu().numpy()
    assert np.array_equal(got[:, 16:16 + c], want) and np.array_equal(steps.cpu().numpy(), wsteps)
    assert np.all(got[:, 16 + c:16 + c8] == 0)                    # zeros behind the row,
    assert np.all(got[:, :16] == 77) and np.all(got[:, 16 + c8:] == 77)      # nothing beyond


def test_row_codes_zeros_behind_infinite_factors(gpu):
    """The zeros behind a row's channels are zeros whatever the factors are."""
    import torch
    f = np.full(136, np.inf, np.float32)
    codes = torch.full((2, 256), 5, dtype=torch.int8, device=gpu)
    tlq.row_codes(dev(np.ones((2, 136)), gpu, "f16"), 8, tlq.params(), codes, torch.empty(2, device=gpu), factor=dev(f, gpu))
    assert bool((codes[:, 136:] == 0).all())


def test_row_codes_of_more_rows_than_a_launch_has_blocks(gpu):
    """Four million rows at once are those of their halves."""
    import torch
    n, p = (1 << 22) + 9, tlq.params()
    X = torch.randn((n, 8), device=gpu).half()
    f = torch.rand(8, device=gpu) + 0.5
    codes, steps = torch.empty((n, 128), dtype=torch.int8, device=gpu), torch.empty(n, device=gpu)
    tlq.row_codes(X, 8, p, codes, steps, factor=f)
    c, s = torch.empty((n // 2 + 1, 128), dtype=torch.int8, device=gpu), torch.empty(n // 2 + 1, device=gpu)
    for r0 in (0, n - n // 2 - 1):
        tlq.row_codes(X[r0:r0 + n // 2 + 1], 8, p, c, s, factor=f)
        assert torch.equal(codes[r0:r0 + n // 2 + 1], c) and torch.equal(steps[r0:r0 + n // 2 + 1], s)


def test_row_codes_of_weights_are_the_channel_quantiser(gpu):
    """The codes are those of fake_quant with symmetric rows."""
    import torch
    g = np.random.default_rng(22)
    W = rnd(g.standard_normal((37, 648)) * 0.02, "f16")
    s = np.exp(g.standard_normal(648)).astype(np.float32)
    p = tlq.params(bits=8, group=0, symmetric=1)
    codes, steps = torch.empty((37, 768), dtype=torch.int8, device=gpu), torch.empty(37, device=gpu)
    tlq.row_codes(dev(W, gpu, "f16"), 8, p, codes, steps, factor=dev(s, gpu))
    stored, delta = torch.empty((37, 648), dtype=torch.uint8, device=gpu), torch.empty((37, 1), device=gpu)
    tlq.fake_quant(dev(W, gpu, "f16"), dev(s, gpu), p, codes=stored, delta=delta)
    assert torch.equal(codes[:, :648].int(), stored.int() - 128) and torch.equal(steps, delta[:, 0])


def _linear_case(g, n, ci, co, dt, bits, wbits=8):
    x = rnd(g.standard_normal((n, ci)) * 2.0, dt)
    x[:, g.integers(0, ci, max(1, ci // 50))] *= 16
    x = rnd(x, dt)
    f = np.exp(0.5 * g.standard_normal(ci)).astype(np.float32)
    wc, ws = ob.row_codes(rnd(g.standard_normal((co, ci)) * 0.03, dt), wbits)
    return x, f, wc, ws


def _padded(wc, gpu, extra=0):
    import torch
    co, ci = wc.shape
    t = torch.zeros((co, -(-ci // 128) * 128 + extra), dtype=torch.int8, device=gpu)
    if extra:
        t[:, -extra:] = 99
    t[:, :ci] = dev(wc, gpu)
    return t


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("out", ["x", "f32"])
@pytest.mark.parametrize("n,ci,co,bits", [
    (1, 8, 1, 8), (1, 4096, 16, 8), (2, 72, 3, 8), (4, 1096, 33, 6), (5, 264, 17, 8), (16, 640, 100, 8), (17, 136, 31, 4),
    (32, 128, 16, 8), (33, 2056, 50, 8), (64, 384, 130, 8), (65, 256, 20, 8), (129, 72, 129, 8), (300, 1096, 263, 6),
    (1, 13824, 24, 8), (3, 11008, 70, 2), (257, 512, 257, 8),
    # tokens shared through LDS: parts of the row of codes and one part, odd numbers of 128 codes, ragged outputs and tokens
    (16, 8200, 9001, 8), (17, 4104, 9001, 8), (40, 2568, 13000, 6), (64, 1096, 20001, 8), (65, 2048, 130, 8), (130, 4104, 1003, 8),
    (256, 2056, 129, 4), (33, 136, 70001, 8),
    # beyond 64 tokens: few outputs, a long row of codes, tiles
    (448, 136, 1009, 8), (65, 2176, 130, 8), (300, 4104, 263, 8), (520, 1096, 1399, 6), (1000, 72, 1003, 8)])
def test_linear_i8(gpu, dt, out, n, ci, co, bits):
    import torch
    g = np.random.default_rng([23, n, ci, co])
    x, f, wc, ws = _linear_case(g, n, ci, co, dt, bits)
    od = dt if out == "x" else "f32"
    p = tlq.params(act_bits=bits, x_dtype=CODE[dt], yref_dtype=CODE[od])
    xt, _ = spread(x, gpu, dt)
    y, wide = spread(np.zeros((n, co), np.float32), gpu, od)
    work = torch.full((tlq.linear_i8_workspace_bytes(n, ci),), 0xAB, dtype=torch.uint8, device=gpu)
    tlq.linear_i8(xt, _padded(wc, gpu, 16), dev(ws, gpu), p, y, factor=dev(f, gpu), workspace=work)
    want = ob.linear_i8(x, bits, wc, ws, f)
    # the sum as a float, two products, the output: each a rounding
    within(host(y), want, np.abs(want) * (HALF[od] + 3.1 * U) + TINY[od] + 1e-44)
    keep = torch.ones(wide.shape[1], dtype=torch.bool)
    keep[8:8 + co] = False
    assert bool((wide[:, keep.to(gpu)] == 3.0).all())


def test_linear_i8_is_the_propagation_of_the_search(gpu):
    """Stored weights and per-token codes give what apply_best gives in the searched setting."""
    import torch
    g = np.random.default_rng(24)
    n, ci, co = 90, 384, 200
    x, W = rnd(g.standard_normal((n, ci)), "bf16"), rnd(g.standard_normal((co, ci)) * 0.02, "bf16")
    s = np.exp(0.5 * g.standard_normal(ci)).astype(np.float32)
    p = tlq.params(bits=8, group=0, symmetric=1, act_bits=8, x_dtype=tlq.BF16, yref_dtype=tlq.BF16)
    X, Wt, st = dev(x, gpu, "bf16"), dev(W, gpu, "bf16"), dev(s, gpu)
    a, y = (torch.empty((n, co), dtype=torch.bfloat16, device=gpu) for _ in range(2))
    tlq.apply_best(X, Wt, st, p, a)
    codes, steps = torch.empty((co, 384), dtype=torch.int8, device=gpu), torch.empty(co, device=gpu)
    tlq.row_codes(Wt, 8, p, codes, steps, factor=st)
    for rows in (n, 20):                                       # large tiles, the kernel for few tokens
        tlq.linear_i8(X[:rows], codes, steps, p, y[:rows], factor=dev(np.float32(1) / s, gpu))
        d = (y[:rows].float() - a[:rows].float()).abs()
        assert bool((d <= 2 * HALF["bf16"] * a[:rows].float().abs() * 1.01).all())    # (either may round the last bit the other way)


def test_linear_i8_extreme_sums(gpu):
    """The largest sums that the codes allow: exact in 32 bits."""
    import torch
    n, ci, co = 2, 65536, 5
    x = np.ones((n, ci), np.float32)
    x[1] = -1.0
    wc, ws = np.full((co, ci), -128, np.int8), np.ones(co, np.float32)
    p = tlq.params(act_bits=8, yref_dtype=tlq.F32)
    for rows in (n, 66):
        X = dev(np.repeat(x, 33, 0)[:rows] if rows > n else x, gpu, "f16")
        y = torch.empty((rows, 8), device=gpu)[:, :co]
        tlq.linear_i8(X, dev(wc, gpu), dev(ws, gpu), p, y)
        want = ob.linear_i8(X.float().cpu().numpy(), 8, wc, ws)
        within(host(y), want, np.abs(want) * 4 * U)


def _kernels(call):
    """Names of the library's launches of a call, other than the codes'."""
    tlq.profile_reset()
    tlq.profile_enable(True)
    try:
        call()
        return {k.name for k in tlq.profile_read() if k.launches} - {"row_codes", "act_quant"}
    finally:
        tlq.profile_enable(False)
        tlq.profile_reset()


FEW, MID, TILES = {"linear_few"}, {"linear_mid", "linear_join"}, {"gemm_store"}


@pytest.mark.parametrize("dt,out", [("f16", "x"), ("bf16", "f32"), ("bf16", "x")])
@pytest.mark.parametrize("n,ci,co,kernels", [
    (300, 1096, 263, FEW), (64, 8200, 2203, MID), (200, 4104, 1003, MID), (300, 4104, 263, TILES),
    # tiles of 128 x 128, at most one a CU and more; of 256 outputs x 256, 192 and 320 tokens; ragged outputs and tokens
    (1000, 264, 2051, TILES), (2501, 136, 2050, TILES), (6391, 136, 2557, TILES), (4001, 136, 2051, TILES), (8001, 136, 2051, TILES),
    # rows longer than the search's
    (300, 20008, 70, TILES), (520, 65536, 262, TILES)])
def test_linear_i8_by_kernel(gpu, dt, out, n, ci, co, kernels):
    """Every kernel of the product, each named, against the oracle."""
    import torch
    g = np.random.default_rng([25, n, ci, co])
    x, f, wc, ws = _linear_case(g, n, ci, co, dt, 8)
    od = dt if out == "x" else "f32"
    p = tlq.params(act_bits=8, x_dtype=CODE[dt], yref_dtype=CODE[od])
    xt, _ = spread(x, gpu, dt)
    y, wide = spread(np.zeros((n, co), np.float32), gpu, od)
    work = torch.full((tlq.linear_i8_workspace_bytes(n, ci),), 0xAB, dtype=torch.uint8, device=gpu)
    w, s, ft = _padded(wc, gpu, 16), dev(ws, gpu), dev(f, gpu)
    assert _kernels(lambda: tlq.linear_i8(xt, w, s, p, y, factor=ft, workspace=work)) == kernels
    want = ob.linear_i8(x, 8, wc, ws, f)
    within(host(y), want, np.abs(want) * (HALF[od] + 3.1 * U) + TINY[od] + 1e-44)
    keep = torch.ones(wide.shape[1], dtype=torch.bool)
    keep[8:8 + co] = False
    assert bool((wide[:, keep.to(gpu)] == 3.0).all())


def test_linear_i8_is_the_propagation_of_the_search_in_every_kernel(gpu):
    """What apply_best gives, by the kernels for few tokens, for shared tokens and by tiles."""
    import torch
    g = np.random.default_rng(26)
    for n, ci, co, cases in ((700, 384, 1003, ((700, TILES), (300, FEW), (20, FEW))), (300, 4104, 200, ((300, TILES), (256, MID), (50, FEW))),
                             (64, 8200, 2400, ((64, MID),))):
        x, W = rnd(g.standard_normal((n, ci)), "bf16"), rnd(g.standard_normal((co, ci)) * 0.02, "bf16")
        s = np.exp(0.5 * g.standard_normal(ci)).astype(np.float32)
        p = tlq.params(bits=8, group=0, symmetric=1, act_bits=8, x_dtype=tlq.BF16, yref_dtype=tlq.BF16)
        X, Wt, st = dev(x, gpu, "bf16"), dev(W, gpu, "bf16"), dev(s, gpu)
        a, y = (torch.empty((n, -(-co // 8) * 8), dtype=torch.bfloat16, device=gpu)[:, :co] for _ in range(2))
        tlq.apply_best(X, Wt, st, p, a)
        codes, steps = torch.empty((co, -(-ci // 128) * 128), dtype=torch.int8, device=gpu), torch.empty(co, device=gpu)
        tlq.row_codes(Wt, 8, p, codes, steps, factor=st)
        inv = dev(np.float32(1) / s, gpu)
        for rows, kernels in cases:
            assert _kernels(lambda: tlq.linear_i8(X[:rows], codes, steps, p, y[:rows], factor=inv)) == kernels, rows
            d = (y[:rows].float() - a[:rows].float()).abs()
            assert bool((d <= 2 * HALF["bf16"] * a[:rows].float().abs() * 1.01).all())    # (either may round the last bit the other way)


@pytest.mark.parametrize("rows,co,kernels", [(300, 5, TILES), (700, 262, TILES), (66, 300, MID)])
def test_linear_i8_extreme_sums_in_tiles(gpu, rows, co, kernels):
    """The largest sums that the codes allow, 2^30, of either sign: exact in 32 bits."""
    import torch
    ci = 65536
    x = torch.ones((rows, ci), dtype=torch.float16, device=gpu)
    x[1::2] = -1.0
    # (127 times -128 each; a token of -1 and weights of 127 to -128 in turn meet the other sign)
    wc = torch.full((co, ci), -128, dtype=torch.int8, device=gpu)
    wc[1::3] = 127
    ws = torch.ones(co, device=gpu)
    p = tlq.params(act_bits=8, yref_dtype=tlq.F32)
    y = torch.empty((rows, -(-co // 8) * 8), device=gpu)[:, :co]
    assert _kernels(lambda: tlq.linear_i8(x, wc, ws, p, y)) == kernels
    row = np.where(np.arange(co) % 3 == 1, 127.0, -128.0) * 127.0 * ci
    want = np.where(np.arange(rows) % 2 == 0, 1.0, -1.0)[:, None] * row[None, :] * float(np.float32(1) / np.float32(127))
    within(host(y), want, np.abs(want) * 4 * U)


# ------------------------------------------------------------------ queries and keys
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,h,kv,dh,rot,pairs,norm,far", [
    (1, 1, 1, 64, 64, False, True, 10), (5, 3, 1, 128, 128, False, True, 5000), (16, 32, 8, 128, 128, False, True, 2 ** 31 - 1),
    (7, 7, 1, 128, 64, False, False, 1000), (33, 5, 5, 256, 256, True, True, 100000), (4, 2, 2, 64, 48, False, True, 77),
    (9, 4, 2, 64, 16, True, False, 3000), (3, 9, 3, 256, 80, False, True, 10 ** 6), (6, 2, 1, 128, 0, False, True, 9),
    (8200, 1, 1, 64, 64, False, True, 9000)])
def test_qk_norm_rope(gpu, dt, n, h, kv, dh, rot, pairs, norm, far):
    import torch
    g = np.random.default_rng([31, n, h, dh, rot])
    q, k = (rnd(g.standard_normal((n, m * dh)) * np.exp(g.standard_normal((n, 1))), dt) for m in (h, kv))
    q[0] = 0.0                                                # a head of zeros stays zeros
    pos = g.integers(0, far, n).astype(np.int32)
    pos[-1] = far if far < 2 ** 31 - 1 else -(2 ** 31)
    inv = 1e6 ** (-np.arange(rot // 2) / max(1, rot // 2))
    w = [np.exp(0.3 * g.standard_normal(dh)).astype(np.float32) if norm else None for _ in range(2)]
    p = tlq.params(x_dtype=CODE[dt])
    qk = np.concatenate([q, k], 1)
    both, _ = spread(qk, gpu, dt)
    qo, qw = spread(np.zeros_like(q), gpu, dt)
    ko, kw = spread(np.zeros_like(k), gpu, dt)
    inv_t = dev(inv, gpu) if rot else None
    tlq.qk_norm_rope(both[:, :h * dh], both[:, h * dh:], dh, dev(pos, gpu), inv_t, p, qo, ko,
                     wq=None if w[0] is None else dev(w[0], gpu), wk=None if w[1] is None else dev(w[1], gpu), norm=norm,
                     interleaved=pairs)
    for x, got, wt in ((q, qo, w[0]), (k, ko, w[1])):
        want = ob.qk_norm_rope(x, dh, pos, inv, wt, 1e-6, norm, pairs)
        u = np.abs(ob.qk_norm_rope(x, dh, pos, inv[:0], wt, 1e-6, norm, pairs)).reshape(n, -1, dh)
        both_of = u.copy()                                    # |u_a| + |u_b| of each pair
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            both_of[:, :, a] = both_of[:, :, b] = u[:, :, a] + u[:, :, b]
        # the norm: dh products summed in any order, a root, a quotient, two products; cosine and sine: a fraction of a turn
        # as a float (2 pi 2^-26), the function's own error (two ulp of 1), the angle in double
        delta = (dh + 8) * U + 2 * np.pi * 2.0 ** -26 + 4 * U + np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -51
        within(host(got).reshape(n, -1, dh), want.reshape(n, -1, dh), both_of * delta + np.abs(want).reshape(n, -1, dh) * HALF[dt] * 1.001 + TINY[dt] * 1.01)
    assert bool((qw[:, :8] == 3.0).all()) and bool((kw[:, 8 + kv * dh:] == 3.0).all())
    # in place: the same bits
    tlq.qk_norm_rope(both[:, :h * dh], both[:, h * dh:], dh, dev(pos, gpu), inv_t, p, both[:, :h * dh], both[:, h * dh:],
                     wq=None if w[0] is None else dev(w[0], gpu), wk=None if w[1] is None else dev(w[1], gpu), norm=norm,
                     interleaved=pairs)
    assert torch.equal(both[:, :h * dh], qo) and torch.equal(both[:, h * dh:], ko)


@pytest.mark.parametrize("dh,rot,pairs", [(64, 64, False), (128, 64, False), (256, 256, True), (128, 128, False)])
def test_qk_norm_of_heads_whose_squares_are_no_floats(gpu, dh, rot, pairs):
    """Heads near bf16's largest and smallest numbers, beside ordinary ones: squares beyond a float's range on either side."""
    g = np.random.default_rng([32, dh])
    n, h = 12, 5
    size = np.concatenate([2.0 ** np.array([120, 64, 63, 50, 0, -40, -50, -75, -110, -126]), [1.0, 1.0]])
    x = rnd(g.standard_normal((n, h * dh)) * size[:, None], "bf16")
    x[10, dh:2 * dh] *= np.float32(2.0 ** 100)                # (one head of a token)
    x[11, :dh] = rnd(x[11, :dh] * np.float32(2.0 ** -120), "bf16")
    x[3, 0] = rnd(np.array([3e38]), "bf16")[0]                # (one channel of a head)
    pos = g.integers(0, 1000, n).astype(np.int32)
    inv = 1e4 ** (-np.arange(rot // 2) / (rot // 2))
    w = np.exp(0.3 * g.standard_normal(dh)).astype(np.float32)
    for eps in (0.0, 1e-6):
        X = dev(x, gpu, "bf16")
        qo, ko = X.clone(), X.clone()
        tlq.qk_norm_rope(X, X, dh, dev(pos, gpu), dev(inv, gpu), tlq.params(x_dtype=tlq.BF16), qo, ko, wq=dev(w, gpu), wk=dev(w, gpu),
                         eps=eps, interleaved=pairs)
        want = ob.qk_norm_rope(x, dh, pos, inv, w, eps, True, pairs).reshape(n, h, dh)
        u = np.abs(ob.qk_norm_rope(x, dh, pos, inv[:0], w, eps)).reshape(n, h, dh)
        both_of = u.copy()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            both_of[:, :, a] = both_of[:, :, b] = u[:, :, a] + u[:, :, b]
        delta = (dh + 8) * U + 2 * np.pi * 2.0 ** -26 + 4 * U + pos[:, None, None] * 2.0 ** -51
        for got in (qo, ko):
            within(host(got).reshape(n, h, dh), want, both_of * delta + np.abs(want) * HALF["bf16"] * 1.001 + 2.0 ** -126 * 1.01)


# ------------------------------------------------------------------ the cache
class Pool:
    """A pool of pages with sequences in it, on the host and on the device."""

    def __init__(self, g, gpu, lens, new, kv, dh, page, dt, spare=2, wild=False):
        self.g, self.gpu, self.dt = g, gpu, dt
        self.new, self.lens, self.kv, self.dh, self.page = list(new), list(lens), kv, dh, page
        need = [-(-max(n, 0) // page) for n in lens]
        self.n = sum(need) + spare
        order = g.permutation(self.n)
        self.table = np.full((len(lens), max(max(need), 1) + 1), -1, np.int32)
        at = 0
        for s, m in enumerate(need):
            self.table[s, :m] = order[at:at + m]
            at += m
        self.kc = np.clip(np.rint(g.standard_normal((self.n, kv, page, dh)) * 40), -127, 127).astype(np.int8)
        self.vc = np.clip(np.rint(g.standard_normal((self.n, kv, dh, page)) * 40), -127, 127).astype(np.int8)
        w = 3.0 if wild else 0.4
        self.ks = (0.02 * np.exp(0.4 * g.standard_normal((self.n, kv)))).astype(np.float32)
        self.vs = (0.02 * np.exp(w * g.standard_normal((self.n, kv)))).astype(np.float32)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.rows = int(self.cu[-1])
        self.max_new, self.max_len = max(max(new), 1), max(max(lens), max(new), 1)

    def load(self):
        d = lambda a: dev(a, self.gpu)
        self.t = (d(self.kc), d(self.ks), d(self.vc), d(self.vs))
        self.l = np.array(self.lens, np.int32)
        return tlq.kv_batch(d(self.cu), d(self.l), d(self.table), self.max_new, self.max_len), tlq.kv_cache(*self.t)


APPENDS = [
    ([1], [1], 1, 64, 16), ([16, 17, 33], [16, 1, 33], 2, 128, 16), ([100, 64, 65, 1], [37, 64, 1, 1], 3, 128, 64),
    ([200, 0, 5], [90, 0, 5], 2, 64, 128), ([300, 299], [3, 299], 1, 128, 256), ([48, 40, 47], [9, 40, 2], 5, 128, 32),
    ([2, 130], [5, 2], 2, 64, 32),           # more new rows than the sequence has tokens
    ([300, 128, 129, 1], [190, 100, 129, 1], 2, 128, 128), ([700, 256, 257, 300], [500, 130, 257, 299], 3, 64, 256),
    ([200, 64], [150, 64], 1, 64, 64), ([90, 33], [80, 20], 2, 64, 32), ([70, 17], [60, 16], 2, 128, 16),
    ([600, 513], [400, 513], 1, 128, 256),
]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,kv,dh,page", APPENDS)
def test_kv_append(gpu, dt, lens, new, kv, dh, page):
    """Codes and steps are those of the definition, bit for bit; what is not written stays as it was."""
    g = np.random.default_rng([41, sum(lens), page, dh])
    c = Pool(g, gpu, lens, new, kv, dh, page, dt)
    rows = c.rows + 3                                         # rows behind the last sequence: no part in anything
    x = rnd(g.standard_normal((rows, 2 * kv * dh)) * np.exp(1.5 * g.standard_normal((rows, 1))), dt)
    x[c.rows:] = np.nan
    x[0, :dh] = 0.0
    b, cache = c.load()
    wide, _ = spread(x, gpu, dt)
    tlq.kv_append(wide[:, :kv * dh], wide[:, kv * dh:], b, cache, tlq.params(x_dtype=CODE[dt]))
    ob.kv_append(x[:, :kv * dh], c.kc, c.ks, c.cu, c.lens, c.table, c.max_len, False)
    ob.kv_append(x[:, kv * dh:], c.vc, c.vs, c.cu, c.lens, c.table, c.max_len, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_kv_append_one_by_one_grows_the_step(gpu):
    """Tokens one at a time, each louder or quieter than the last: earlier codes follow the page's step."""
    g = np.random.default_rng(42)
    kv, dh, page, dt = 2, 64, 16, "bf16"
    c = Pool(g, gpu, [20], [20], kv, dh, page, dt)
    x = rnd(g.standard_normal((20, kv * dh)) * np.array([1, 3, 0.1, 50, 2] * 4)[:, None], dt)
    b, cache = c.load()
    X = dev(x, gpu, dt)
    one = np.array([0, 1], np.int32)
    for t in range(20):
        lens = np.array([t + 1], np.int32)
        tlq.kv_append(X[t:t + 1], X[t:t + 1], tlq.kv_batch(dev(one, gpu), dev(lens, gpu), b.parts[2], 1, 32), cache, tlq.params(x_dtype=tlq.BF16))
        ob.kv_append(x[t:t + 1], c.kc, c.ks, one, lens, c.table, 32, False)
        ob.kv_append(x[t:t + 1], c.vc, c.vs, one, lens, c.table, 32, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_kv_append_of_infinities_and_nan(gpu):
    g = np.random.default_rng(43)
    c = Pool(g, gpu, [24], [20], 1, 64, 16, "f16")
    x = rnd(g.standard_normal((20, 64)), "f16")
    x[3, 5], x[4, 6], x[5, 7], x[19, :] = np.inf, -np.inf, np.nan, np.nan
    b, cache = c.load()
    X = dev(x, gpu, "f16")
    tlq.kv_append(X, X, b, cache, tlq.params())
    ob.kv_append(x, c.kc, c.ks, c.cu, c.lens, c.table, c.max_len, False)
    ob.kv_append(x, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def _attend(gpu, c, heads, dt, q, scale=0.0, rows=None, poison=True):
    import torch
    b, cache = c.load()
    wide_q, _ = spread(q, gpu, dt)
    out, wide = spread(np.zeros_like(q), gpu, dt)
    wide.fill_(3.0)
    p = tlq.params(x_dtype=CODE[dt])
    work = torch.full((max(256, tlq.kv_attention_workspace_bytes(q.shape[0], heads, b, cache)),), 0xFF, dtype=torch.uint8, device=gpu)
    tlq.kv_attention(wide_q, heads, b, cache, p, out, scale=scale, workspace=work)
    torch.cuda.synchronize()
    got = host(wide)
    assert np.all(got[:, :8] == 3.0) and np.all(got[:, 8 + q.shape[1]:] == 3.0)
    return got[:, 8:8 + q.shape[1]]


def _bounds(c, heads, q, kind):
    """Host's bounds under which the tiles of 128 rows are taken (they need work for many blocks): rows behind the last sequence
    ("tiles"), or, for more than 16 rows, longer sequences than there are ("parts": many parts, most of them empty)."""
    group, pairs = heads // c.kv, len(c.lens) * c.kv
    if kind == "tiles":
        q = np.concatenate([q, np.full((1540 * 16 // (group * pairs) + 16, q.shape[1]), np.nan)])
        c.max_new = q.shape[0]
        c.max_len = max(c.max_len, c.max_new)
    if kind == "parts":
        units = 1540 // (max(-(-c.max_new * group // 16), 1) * pairs) + 1
        c.max_len = max(c.max_len, units * 256)
        c.table = np.concatenate([c.table, np.full((len(c.lens), max(0, -(-c.max_len // c.page) - c.table.shape[1])), -1, np.int32)], 1)
    return q


def _check_attention(gpu, c, heads, dt, q, scale=0.0):
    got = _attend(gpu, c, heads, dt, q, scale)
    want, mag, sens = ob.kv_attention(q, heads, c.kc, c.ks, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len, scale or None)
    none = np.isnan(want[:, 0])
    assert np.all(got[none] == 3.0)                            # rows behind the last sequence stay as they were
    got, want, mag, sens = got[~none], want[~none], mag[~none], np.repeat(sens[~none], c.dh, 1)
    lost = np.isnan(want)                                      # (of a query that is not finite)
    assert np.isnan(got[lost]).all()
    got, want, mag, sens = got[~lost], want[~lost], mag[~lost], sens[~lost]
    # weights in 16 bits, above the line and below it: sum_j p_j e_j (v_j - out), |e_j| <= 2^-11, at most 2^-11 (mag + |out|);
    # those below 2^-21 of the largest to 2^-32 of it; scores as sums of dh products (a relative error of e^(2 ds) in p and in
    # the sum of p), sums over the keys in 32 bits, the output
    n = min(c.max_len, max(c.lens))
    ds = ((c.dh + 6) * sens + 64) * U
    bound = (mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + (n / 4 + 64) * U) + n * 2.0 ** -32 * 127 * c.vs.max() + np.abs(want) * HALF[dt] * 1.001 + TINY[dt] * 1.01
    within(got, want, bound)
    # well inside on average: the weights' roundings do not line up
    assert np.abs(got - want).mean() <= 0.6 * bound.mean()


ATTENTION = [   # lens, new, kv heads, group, dh, page
    ([1], [1], 1, 1, 64, 16), ([1, 2, 3], [1, 1, 1], 2, 2, 128, 16), ([70, 16, 129], [1, 1, 1], 2, 7, 128, 16),
    ([300, 255, 256, 257], [1, 1, 1, 1], 1, 8, 128, 64), ([1000], [1], 3, 4, 64, 32), ([2600, 40], [1, 1], 2, 4, 128, 256),
    ([40, 41, 64], [3, 9, 2], 2, 3, 128, 32), ([65, 130], [65, 130], 2, 1, 128, 64), ([33, 100], [33, 50], 1, 4, 64, 16),
    ([500], [129], 2, 1, 128, 64), ([700, 300, 5], [200, 300, 5], 1, 2, 64, 128), ([150, 0, 20], [150, 0, 20], 2, 6, 128, 16),
    ([1500], [17], 1, 1, 128, 64), ([20], [20], 1, 40, 64, 16),
    ([2600, 700, 30], [40, 40, 30], 2, 3, 128, 32), ([2600, 700, 30], [40, 40, 30], 2, 3, 64, 256),   # splits that some lack
    ([90, 10, 200, 33, 64], [90, 10, 150, 33, 1], 5, 2, 128, 16),                                      # 25 pairs
    ([300] * 3, [140, 1, 300], 3, 1, 64, 16), ([1100, 1024, 513, 256], [1, 1, 1, 1], 1, 16, 64, 16),
]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("lens,new,kv,group,dh,page", ATTENTION)
def test_kv_attention(gpu, dt, kind, lens, new, kv, group, dh, page):
    g = np.random.default_rng([51, sum(lens), group, dh])
    c = Pool(g, gpu, lens, new, kv, dh, page, dt)
    q = rnd(1.5 * g.standard_normal((c.rows + 2, kv * group * dh)), dt)
    q[c.rows:] = np.nan
    _check_attention(gpu, c, kv * group, dt, _bounds(c, kv * group, q, kind))


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_kv_attention_of_wild_steps_and_loud_queries(gpu, dt, kind):
    """Pages whose steps lie five orders of magnitude apart; queries of very different size, zeros among them; scores large
    enough that one key has nearly all of the weight; a scale of the caller's."""
    g = np.random.default_rng(52)
    c = Pool(g, gpu, [400, 333, 90], [1, 6, 90], 2, 128, 16, dt, wild=True)
    q = rnd(g.standard_normal((c.rows, 4 * 128)) * np.exp(2 * g.standard_normal((c.rows, 1))), dt)
    q[2] = 0.0
    if dt == "bf16":
        q[3] = rnd(q[3] * 2.0 ** -100, dt)
    q = _bounds(c, 4, q, kind)
    _check_attention(gpu, c, 4, dt, q)
    _check_attention(gpu, c, 4, dt, q, scale=-0.31)
    c.ks[:] *= 20
    _check_attention(gpu, c, 4, dt, q)


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
def test_kv_attention_of_pages_that_are_not_there(gpu, kind):
    """Entries outside the pool stand for tokens that do not exist, wherever they are; a row that sees none gives zeros; steps and
    codes of pages that no sequence names are never used."""
    g = np.random.default_rng(53)
    for dt, new in (("f16", [1, 3, 1, 2, 70]), ("bf16", [70, 40, 20, 30, 64])):
        c = Pool(g, gpu, [130, 100, 20, 40, 70], new, 2, 128, 16, dt)
        c.table[0, 2], c.table[0, 5], c.table[1, 6], c.table[2, :], c.table[3, 0], c.table[4, :4] = -1, c.n, 2 ** 31 - 1, -5, -(2 ** 31), -1
        named = {int(i) for i in c.table.ravel() if 0 <= i < c.n}
        for i in set(range(c.n)) - named:
            c.ks[i], c.vs[i] = np.nan, np.inf
        q = _bounds(c, 4, rnd(g.standard_normal((c.rows, 4 * 128)), dt), kind)
        keep = c.vs.copy()
        c.vs[~np.isfinite(c.vs)] = 0.0                        # (the bound takes the largest step; put back below)
        top = c.vs.max()
        c.vs = keep
        got = _attend(gpu, c, 4, dt, q)
        assert (got[c.rows:] == 3.0).all()
        want, mag, sens = ob.kv_attention(q, 4, c.kc, c.ks, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len)
        got, want, mag, sens = (t[:c.rows] for t in (got, want, mag, sens))
        ds = ((128 + 6) * np.repeat(sens, 128, 1) + 64) * U
        within(got, want, (mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + 200 * U) + 200 * 2.0 ** -32 * 127 * top + np.abs(want) * HALF[dt] * 1.001 + TINY[dt] * 1.01)
        assert (want == 0).all(axis=1).any()


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("page,dh", [(16, 128), (16, 64), (32, 128)])
def test_kv_attention_of_pages_named_ahead(gpu, kind, dt, page, dh):
    """Pages that the table names behind a sequence's last token, never written: their steps have no part in anything."""
    g = np.random.default_rng([67, page, dh])
    lens, new = [33, 70, 17, 272, 300], [33, 50, 1, 20, 16]
    c = Pool(g, gpu, lens, new, 2, dh, page, dt, spare=8)
    c.table = np.concatenate([c.table, np.full((5, 4), -1, np.int32)], 1)
    spare = [i for i in range(c.n) if i not in set(c.table.ravel().tolist())]
    q = _bounds(c, 4, rnd(g.standard_normal((c.rows, 4 * dh)), dt), kind)
    want = _attend(gpu, c, 4, dt, q)
    assert np.isfinite(want).all()
    for s, n in enumerate(lens):
        c.table[s, -(-n // page):][:4] = np.array(spare)[[s, (s + 3) % 8, 0, 1]]
    for k, v in ((np.nan, np.inf), (np.inf, np.nan), (0.0, np.inf), (np.inf, 0.0), (-1.0, -np.inf), (3e38, 3e38)):
        c.ks[spare], c.vs[spare] = np.float32(k), np.float32(v)
        assert np.array_equal(_attend(gpu, c, 4, dt, q), want), (k, v)


def test_kv_lengths_that_no_batch_should_have(gpu):
    """Lengths beyond the table, beyond the host's bound, negative ones and new rows beyond a length: held to what is there."""
    g = np.random.default_rng(54)
    dt = "bf16"
    c = Pool(g, gpu, [40, 40, 40, 40], [2, 40, 3, 2], 1, 64, 16, dt)
    c.table = c.table[:, :3].copy()                           # 48 tokens a sequence at most
    c.lens = [1000, 25, -7, 40]
    c.max_len = 47
    q = rnd(g.standard_normal((c.rows, 128)), dt)
    _check_attention(gpu, c, 2, dt, q)
    x = rnd(g.standard_normal((c.rows, 64)), dt)
    b, cache = c.load()
    tlq.kv_append(dev(x, gpu, dt), dev(x, gpu, dt), b, cache, tlq.params(x_dtype=tlq.BF16))
    ob.kv_append(x, c.kc, c.ks, c.cu, c.lens, c.table, c.max_len, False)
    ob.kv_append(x, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,most,group,page,kind", [
    ([40, 30], [5, 3], 1, 1, 16, ""), ([700, 40], [5, 20], 3, 2, 16, ""), ([3000, 2], [9, 2], 1, 4, 64, ""),
    ([300, 260, 9], [150, 260, 9], 40, 1, 64, "parts"), ([1500, 30], [200, 7], 130, 2, 32, "parts"), ([90, 70], [70, 70], 17, 2, 128, ""),
    ([10, 33], [20, 33], 12, 1, 16, "")])                    # (the first with rows before its first token)
def test_kv_more_new_tokens_than_the_hosts_bound(gpu, dt, lens, new, most, group, page, kind):
    """Tokens behind a sequence's first max_new: their rows of Out stay as they were, the cache takes none of them."""
    g = np.random.default_rng([68, sum(lens), most])
    c = Pool(g, gpu, lens, new, 2, 64, page, dt)
    heads = 2 * group
    q = rnd(g.standard_normal((c.rows, heads * 64)), dt)
    whole = _attend(gpu, c, heads, dt, q)
    c.max_new = most
    if kind == "parts":
        q = _bounds(c, heads, q, kind)
    got = _attend(gpu, c, heads, dt, q)
    taken = np.concatenate([np.arange(n) < most for n in new])
    assert (got[~taken] == 3.0).all() and not (got[taken] == 3.0).all(axis=1).any()
    want, mag, sens = ob.kv_attention(q, heads, c.kc, c.ks, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len)
    ds = ((64 + 6) * np.repeat(sens, 64, 1) + 64) * U
    n = max(lens)
    bound = (mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + (n / 4 + 64) * U) + n * 2.0 ** -32 * 127 * c.vs.max() + np.abs(want) * HALF[dt] * 1.01 + TINY[dt] * 1.01
    within(got[taken], want[taken], bound[taken])
    within(got[taken], whole[taken], 2 * bound[taken])
    # the oracle's append of the first max_new of each alone
    rows = np.flatnonzero(taken)
    x = rnd(g.standard_normal((c.rows, 2 * 64)), dt)
    b, cache = c.load()
    tlq.kv_append(dev(x, gpu, dt), dev(x, gpu, dt), b, cache, tlq.params(x_dtype=CODE[dt]))
    cu = np.concatenate([[0], np.cumsum(np.minimum(new, most))]).astype(np.int32)
    end = [n - m + min(m, most) for n, m in zip(lens, new)]
    ob.kv_append(x[rows], c.kc, c.ks, cu, end, c.table, c.max_len, False)
    ob.kv_append(x[rows], c.vc, c.vs, cu, end, c.table, c.max_len, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_kv_attention_of_a_shared_prefix(gpu):
    """Two sequences that hold the same first pages give what they give alone."""
    import torch
    g = np.random.default_rng(55)
    c = Pool(g, gpu, [100, 90], [1, 1], 2, 128, 32, "f16")
    c.table[1, :2] = c.table[0, :2]
    q = rnd(g.standard_normal((2, 4 * 128)), "f16")
    _check_attention(gpu, c, 4, "f16", q)


@pytest.mark.parametrize("lens,new", [([700, 90], [1, 1]), ([700, 90], [40, 90])])
def test_kv_tables_that_are_part_of_a_wider_one(gpu, lens, new):
    """Rows of a table further apart than they are long, what lies between them naming pages of no sequence."""
    g = np.random.default_rng(60)
    dt = "bf16"
    c = Pool(g, gpu, lens, new, 2, 128, 64, dt)
    q = rnd(g.standard_normal((c.rows, 4 * 128)), dt)
    x = rnd(g.standard_normal((c.rows, 2 * 128)), dt)
    narrow = _attend(gpu, c, 4, dt, q)
    b, cache = c.load()
    wide = dev(np.concatenate([c.table, np.full((2, 5), c.n - 1, np.int32)], 1), gpu)
    b = tlq.kv_batch(b.parts[0], b.parts[1], wide[:, :c.table.shape[1]], c.max_new, c.max_len)
    Q, X, p = dev(q, gpu, dt), dev(x, gpu, dt), tlq.params(x_dtype=CODE[dt])
    assert np.array_equal(host(tlq.kv_attention(Q, 4, b, cache, p, dev(q, gpu, dt))), narrow)
    tlq.kv_append(X, X, b, cache, p)
    ob.kv_append(x, c.kc, c.ks, c.cu, c.lens, c.table, c.max_len, False)
    ob.kv_append(x, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len, True)
    for got, want in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_kv_attention_of_very_many_sequences(gpu):
    """More blocks than one row of a grid has here, nearly all of them of sequences without tokens."""
    g = np.random.default_rng(62)
    lens, new = np.zeros(65535, np.int64), np.zeros(65535, np.int64)
    lens[[0, 40000, 65527, 65534]], new[[0, 40000, 65527, 65534]] = [70, 33, 20, 150], [70, 1, 20, 20]
    c = Pool(g, gpu, lens.tolist(), new.tolist(), 1, 64, 16, "f16")
    q = np.full((2300, 64), np.nan, np.float32)                # (18 tiles a sequence by the host's bound)
    q[:c.rows] = rnd(g.standard_normal((c.rows, 64)), "f16")
    c.max_new, c.max_len = 2300, 2300
    _check_attention(gpu, c, 1, "f16", q)


def test_kv_attention_of_more_splits_than_lanes(gpu):
    """Parts of 256 keys of one sequence, and of a short one beside it."""
    g = np.random.default_rng(61)
    c = Pool(g, gpu, [40000, 300], [1, 1], 1, 128, 128, "bf16")
    _check_attention(gpu, c, 4, "bf16", rnd(g.standard_normal((2, 4 * 128)), "bf16"))


def test_kv_pools_beyond_two_to_the_31(gpu):
    """Pages whose codes lie further than 2^31 and 2^32 bytes into the pool."""
    import torch
    kv, dh, page, n = 2, 128, 256, (1 << 16) + 300            # 65,536 bytes a page: 4.3 GB of keys, as many of values
    kc, vc = (torch.empty((n, kv) + sh, dtype=torch.int8, device=gpu) for sh in ((page, dh), (dh, page)))
    ks, vs = (torch.empty((n, kv), dtype=torch.float32, device=gpu) for _ in range(2))
    cache = tlq.kv_cache(kc, ks, vc, vs)
    small = [t[:8].clone() for t in (kc, ks, vc, vs)]
    near = tlq.kv_cache(*small)
    far = np.array([[n - 1, 40000, 5], [65537, 32769, 3]], np.int32)
    cu, lens = np.array([0, 600, 1100], np.int32), np.array([600, 500], np.int32)
    X = torch.randn((1100, kv * dh), device=gpu).half()
    p = tlq.params()
    outs = []
    for table, pool in ((far, cache), (np.array([[0, 1, 2], [3, 4, 5]], np.int32), near)):
        t = dev(table, gpu)
        tlq.kv_append(X, X, tlq.kv_batch(dev(cu, gpu), dev(lens, gpu), t, 600, 600), pool, p)
        Q = X.repeat(1, 2).contiguous()
        outs.append(tlq.kv_attention(Q, 4, tlq.kv_batch(dev(cu, gpu), dev(lens, gpu), t, 600, 600), pool, p, torch.empty_like(Q)))
        one = tlq.kv_batch(dev(np.array([0, 1, 2], np.int32), gpu), dev(lens, gpu), t, 1, 600)
        tlq.kv_append(X[:2], X[2:4], one, pool, p)            # (the few-token kernels)
        outs.append(tlq.kv_attention(Q[:2], 4, one, pool, p, torch.empty_like(Q[:2])))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    assert outs[0].isfinite().all() and outs[1].isfinite().all()


def test_kv_attention_of_a_long_sequence(gpu):
    """40,000 keys of which a few have most of the weight: what lies far below them still counts."""
    g = np.random.default_rng(56)
    c = Pool(g, gpu, [40001], [1], 1, 64, 64, "f16")
    q = rnd(2.0 * g.standard_normal((1, 2 * 64)), "f16")
    _check_attention(gpu, c, 2, "f16", q)
    # one key 2^17 times as heavy as each of the others: together they have a quarter of the weight
    c.kc[:] = 0
    c.kc[c.table[0, 300], 0, 5, :] = 127
    c.ks[:] = np.float32(17 * np.log(2) / (127 * 8))
    _check_attention(gpu, c, 2, "f16", np.ones((1, 128), np.float32))


@pytest.mark.parametrize("new,kind", [(1, ""), (20, ""), (20, "tiles"), (20, "parts")])
@pytest.mark.parametrize("dt,length,page,at,heavy,high,low", [
    # one key of the page with values has half of the weight, zeros elsewhere (the step that an append gives them)
    ("f16", 4096, 64, 0, True, 30 / 127, 1e-5 / 127), ("f16", 4096, 64, 40, True, 4 / 127, 1e-5 / 127),
    # equal scores: a page of zeros, or all but one, beside pages with values up to the type's largest; few keys, and many
    ("f16", 32, 16, 0, False, 1000 / 127, 1e-5 / 127), ("f16", 32, 16, 1, False, 16000 / 127, 1e-5 / 127),
    ("f16", 200, 16, 5, False, 65504 / 127, 1e-5 / 127), ("bf16", 3000, 32, 90, False, 1e6, 1e-5 / 127),
    ("bf16", 40000, 64, 0, True, 0.3, 1e-3 / 127), ("f16", 40000, 64, 600, True, 500.0, 1e-3 / 127),
    # further apart than a float's exponents, in one part of the keys and in two; a step of zero
    ("bf16", 200, 16, 0, False, 2.0 ** 118, 2.0 ** -60), ("bf16", 3000, 64, 45, False, 2.0 ** 118, 2.0 ** -60),
    ("bf16", 3000, 64, 0, False, 2.0 ** 118, 2.0 ** -60), ("f16", 600, 64, 3, False, 0.02, 0.0)])
def test_kv_attention_of_quiet_pages_beside_a_loud_one(gpu, new, kind, dt, length, page, at, heavy, high, low):
    """Keys whose values have a step far below that of the loudest page count in the softmax's sum with all of their weight."""
    g = np.random.default_rng([66, length, at])
    c = Pool(g, gpu, [length + new - 1], [new], 1, 64, page, dt)
    c.vs[:] = np.float32(low)
    c.vs[c.table[0, at]] = np.float32(high)
    c.vc[c.table[0, at]] = np.abs(c.vc[c.table[0, at]])      # (their mean is no zero)
    if heavy:
        c.kc[:] = 0
        c.kc[c.table[0, at], 0, 5, :] = 127
        c.ks[:] = np.float32(np.log(length) / (127 * 8))
        q = np.ones((new, 128), np.float32)
    else:
        q = rnd(0.1 * g.standard_normal((new, 128)), dt)
    got = _attend(gpu, c, 2, dt, _bounds(c, 2, q, kind))[:new]
    want, mag, sens = ob.kv_attention(q, 2, c.kc, c.ks, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len)
    # as in _check_attention; the sum of the weights may lose 2^-14 of itself and 2^-29 for each key
    ds = ((64 + 6) * np.repeat(sens, 64, 1) + 64) * U
    n = length + new
    bound = ((mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + (n / 4 + 64) * U) + n * 2.0 ** -32 * 127 * c.vs.max() +
             np.abs(want) * (2.0 ** -14 + n * 2.0 ** -29 + HALF[dt] * 1.001) + TINY[dt] * 1.01)
    within(got, want, bound)


@pytest.mark.parametrize("new,kind", [(1, ""), (20, ""), (20, "tiles"), (20, "parts")])
def test_kv_attention_of_many_keys_far_below_one(gpu, new, kind):
    """One key 2^22 times as heavy as each of 40,000 others, whose weights are no normal halves: together one percent of the sum,
    in the numerator and in the denominator alike."""
    g = np.random.default_rng(57)
    c = Pool(g, gpu, [40000 + new], [new], 1, 64, 64, "f16")
    for page in (2, 300, 600):                               # the heavy key in front, in the middle, near the end
        c.kc[:] = 0
        c.kc[c.table[0, page], 0, 5, :] = 127
        c.ks[:] = np.float32(22 * np.log(2) / (127 * 8))
        c.vc[c.table[0, page], 0, :, 5] = 0                  # what is left is the others' alone
        c.vc[:] = np.abs(c.vc)
        c.vs[:] = np.float32(0.03)
        got = _attend(gpu, c, 2, "f16", _bounds(c, 2, np.ones((new, 128), np.float32), kind))[:new]
        want, mag, _ = ob.kv_attention(np.ones((new, 128)), 2, c.kc, c.ks, c.vc, c.vs, c.cu, c.lens, c.table, c.max_len)
        # weights of 2^-15 and 2^7, exact halves; the score to 2^-17 of itself, sums in 32 bits, a half of a small output
        within(got, want, want * (22 * 64 * U + 2.0 ** -11 * 1.01 + 40000 / 16 * U) + TINY["f16"])


def test_kv_attention_of_queries_near_the_types_largest(gpu):
    """bf16 queries of 2^127 and more against keys as small as that they give ordinary scores; subnormal ones."""
    g = np.random.default_rng(58)
    c = Pool(g, gpu, [70, 300], [2, 30], 1, 128, 16, "bf16")
    c.ks *= np.float32(2.0 ** -122)
    q = rnd(g.standard_normal((c.rows, 256)), "bf16")
    with np.errstate(over="ignore"):                         # (a number above 4 ends as an infinity: NaN for its head)
        q = rnd(np.float32(2.0 ** 126) * q / np.abs(q).max(axis=1, keepdims=True) * 3.9, "bf16")
    assert np.isfinite(q).mean() > 0.99
    _check_attention(gpu, c, 2, "bf16", q)
    c.ks *= np.float32(2.0 ** 122)
    _check_attention(gpu, c, 2, "bf16", rnd(q.astype(np.float64) * 2.0 ** -258, "bf16"))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new,kind", [(1, ""), (20, ""), (20, "tiles"), (20, "parts"), (150, ""), (150, "tiles"), (150, "parts")])
def test_kv_attention_of_queries_that_are_not_finite(gpu, dt, new, kind):
    """An infinity or a NaN anywhere in a query makes its head NaN, whichever sign the keys have there, and no other head; a row
    that sees no key gives zeros still.  Split and unsplit."""
    g = np.random.default_rng(59)
    for length in (200, 3000):
        c = Pool(g, gpu, [length, 40], [new, 1], 2, 64, 32, dt)
        c.kc[:, 0] = np.abs(c.kc[:, 0])
        c.table[1, :] = -1
        q = _bounds(c, 4, rnd(g.standard_normal((c.rows, 4 * 64)), dt), kind)
        clean = _attend(gpu, c, 4, dt, q)
        bad = q.copy()
        bad[0, 3], bad[0, 64 * 2 + 50] = -np.inf, np.nan       # heads 0 and 2
        bad[new // 2, 64 + 63], bad[new // 2, 64 * 3] = np.inf, -np.inf
        bad[c.rows - 1, 0] = np.nan
        got = _attend(gpu, c, 4, dt, bad)
        lost = np.repeat(~np.isfinite(bad).reshape(len(bad), 4, 64).all(2), 64, 1)
        lost[c.rows - 1:] = False                              # (rows behind the last sequence stay as they were)
        assert np.isfinite(clean).all() and (clean[c.rows - 1] == 0.0).all()
        assert np.isnan(got[lost]).all() and np.array_equal(got[~lost], clean[~lost])


# ------------------------------------------------------------------ together
def _block(gpu, g, d, heads, kv, dh, ffn, dt):
    """Weights of a block as stored codes and steps, and its vectors."""
    import torch
    out = {}
    for name, co, ci in (("qkv", (heads + 2 * kv) * dh, d), ("o", d, heads * dh), ("gate_up", 2 * ffn, d), ("down", d, ffn)):
        W = dev(rnd(g.standard_normal((co, ci)) * ci ** -0.5, dt), gpu, dt)
        s = np.exp(0.3 * g.standard_normal(ci)).astype(np.float32)
        codes = torch.empty((co, -(-ci // 128) * 128), dtype=torch.int8, device=gpu)
        steps = torch.empty(co, device=gpu)
        tlq.row_codes(W, 8, tlq.params(x_dtype=CODE[dt]), codes, steps, factor=dev(s, gpu))
        out[name] = (codes, steps, dev(np.float32(1) / s, gpu))
    return out


@pytest.mark.parametrize("dt,heads,kv,dh", [("bf16", 4, 2, 128), ("f16", 6, 1, 64)])
def test_a_block_in_eight_bits(gpu, dt, heads, kv, dh):
    """Prompts of three sequences and four steps of single tokens through a whole block, as a program runs it; every operator
    is held to the oracle on the inputs that it met."""
    import torch
    g = np.random.default_rng([61, heads])
    d, ffn, page = 256, 384, 16
    w = _block(gpu, g, d, heads, kv, dh, ffn, dt)
    p = tlq.params(bits=8, group=0, symmetric=1, act_bits=8, x_dtype=CODE[dt], yref_dtype=CODE[dt])
    inv = 1e4 ** (-np.arange(dh // 2) / (dh // 2))
    wq, wk = (np.exp(0.2 * g.standard_normal(dh)).astype(np.float32) for _ in range(2))
    prompt = [19, 33, 7]
    c = Pool(g, gpu, [n + 4 for n in prompt], prompt, kv, dh, page, dt)
    c.load()
    cache = tlq.kv_cache(*c.t)
    table = dev(c.table, gpu)
    lens = np.zeros(3, np.int32)
    new = lambda n, m: torch.empty((n, m), dtype=tt(dt), device=gpu)

    def linear(x, name):
        codes, steps, f = w[name]
        y = tlq.linear_i8(x, codes, steps, p, new(x.shape[0], codes.shape[0]), factor=f)
        want = ob.linear_i8(host(x), 8, codes[:, :x.shape[1]].cpu().numpy(), steps.cpu().numpy(), f.cpu().numpy())
        within(host(y), want, np.abs(want) * (HALF[dt] + 3.1 * U) + TINY[dt])
        return y

    for counts in [prompt] + [[1, 1, 1]] * 4:
        n = sum(counts)
        lens = lens + np.array(counts, np.int32)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        pos = np.concatenate([np.arange(l - m, l) for l, m in zip(lens, counts)]).astype(np.int32)
        batch = tlq.kv_batch(dev(cu, gpu), dev(lens.astype(np.int32), gpu), table, max(counts), 64)
        h = dev(rnd(g.standard_normal((n, d)), dt), gpu, dt)
        qkv = linear(tlq.rmsnorm_mul(h, p, new(n, d)), "qkv")
        q, k, v = qkv[:, :heads * dh], qkv[:, heads * dh:(heads + kv) * dh], qkv[:, (heads + kv) * dh:]
        before = host(q)
        tlq.qk_norm_rope(q, k, dh, dev(pos, gpu), dev(inv, gpu), p, q, k, wq=dev(wq, gpu), wk=dev(wk, gpu))
        want = ob.qk_norm_rope(before, dh, pos, inv, wq)
        within(host(q), want, np.abs(want) * HALF[dt] * 1.001 + 2e-5 * np.abs(want).max())
        tlq.kv_append(k, v, batch, cache, p)
        ob.kv_append(host(k), c.kc, c.ks, cu, lens, c.table, 64, False)
        ob.kv_append(host(v), c.vc, c.vs, cu, lens, c.table, 64, True)
        for got, code in zip(c.t, (c.kc, c.ks, c.vc, c.vs)):
            assert np.array_equal(got.cpu().numpy(), code)
        a = tlq.kv_attention(q, heads, batch, cache, p, new(n, heads * dh))
        want, mag, sens = ob.kv_attention(host(q), heads, c.kc, c.ks, c.vc, c.vs, cu, lens, c.table, 64)
        ds = ((dh + 6) * np.repeat(sens, dh, 1) + 64) * U
        within(host(a), want, (mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + 100 * U) + np.abs(want) * HALF[dt] * 1.001 + TINY[dt] + 1e-7)
        h = tlq.residual_add(h, linear(a, "o"), p, h)
        gu = linear(tlq.rmsnorm_mul(h, p, new(n, d)), "gate_up")
        m = tlq.silu_mul(gu[:, :ffn], gu[:, ffn:], p, new(n, ffn))
        h = tlq.residual_add(h, linear(m, "down"), p, h)
        assert bool(torch.isfinite(h).all())


def test_a_step_as_a_graph(gpu):
    """One step of single tokens captured; lengths and inputs change between replays, eager work lies between them, and a second
    graph shares the workspace."""
    import torch
    g = np.random.default_rng(62)
    heads, kv, dh, page, dt = 8, 2, 128, 64, "bf16"
    d = heads * dh
    p = tlq.params(act_bits=8, x_dtype=tlq.BF16, yref_dtype=tlq.BF16)
    c = Pool(g, gpu, [900, 700], [1, 1], kv, dh, page, dt)
    c.load()
    cache = tlq.kv_cache(*c.t)
    w = _block(gpu, g, d, heads, kv, dh, 128, dt)
    cu, lens, table = dev(c.cu, gpu), dev(np.array([700, 500], np.int32), gpu), dev(c.table, gpu)
    pos = torch.zeros(2, dtype=torch.int32, device=gpu)
    inv = dev(1e4 ** (-np.arange(64) / 64.0), gpu)
    batch = tlq.kv_batch(cu, lens, table, 1, 900)
    h = torch.empty((2, d), dtype=tt(dt), device=gpu)
    qkv = torch.empty((2, (heads + 2 * kv) * dh), dtype=tt(dt), device=gpu)
    a, y = torch.empty_like(h), torch.empty_like(h)
    ws = torch.empty(max(tlq.linear_i8_workspace_bytes(2, d), tlq.kv_attention_workspace_bytes(2, heads, batch, cache)), dtype=torch.uint8, device=gpu)

    def step(out):
        codes, steps, f = w["qkv"]
        tlq.linear_i8(h, codes, steps, p, qkv, factor=f, workspace=ws)
        q, k, v = qkv[:, :d], qkv[:, d:d + kv * dh], qkv[:, d + kv * dh:]
        tlq.qk_norm_rope(q, k, dh, pos, inv, p, q, k)
        tlq.kv_append(k, v, batch, cache, p)
        tlq.kv_attention(q, heads, batch, cache, p, a, workspace=ws)
        codes, steps, f = w["o"]
        tlq.linear_i8(a, codes, steps, p, out, factor=f, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h.copy_(dev(rnd(g.standard_normal((2, d)), dt), gpu, dt))
        step(y)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    y2 = torch.empty_like(y)
    graphs = []
    for out in (y, y2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            step(out)
    saved = [t.clone() for t in c.t]
    for i in range(4):
        h.copy_(dev(rnd(g.standard_normal((2, d)), dt), gpu, dt))
        lens.copy_(dev(np.array([701 + 60 * i, 501 + i], np.int32), gpu))
        pos.copy_(lens - 1)
        for t, o in zip(c.t, saved):
            t.copy_(o)
        step(y)
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, a, *c.t)]
        for graph, out in zip(graphs, (y, y2)):
            for t, o in zip(c.t, saved):
                t.copy_(o)
            ws.fill_(0xFF)
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for got, e in zip((out, a, *c.t), want):
                assert torch.equal(got, e)


def test_calls_on_another_stream(gpu):
    """The calls run on the current stream, in its order."""
    import torch
    g = np.random.default_rng(63)
    c = Pool(g, gpu, [200], [1], 2, 128, 16, "f16")
    b, cache = c.load()
    q = dev(rnd(g.standard_normal((1, 512)), "f16"), gpu, "f16")
    k = dev(rnd(g.standard_normal((1, 256)), "f16"), gpu, "f16")
    p = tlq.params()
    saved = [t.clone() for t in c.t]
    tlq.kv_append(k, k, b, cache, p)
    want = tlq.kv_attention(q, 4, b, cache, p, torch.empty_like(q)).clone()
    for t, o in zip(c.t, saved):
        t.copy_(o)
    out, late = torch.zeros_like(q), torch.zeros_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late.copy_(k)
        tlq.kv_append(late, late, b, cache, p)
        tlq.kv_attention(q, 4, b, cache, p, out)
    side.synchronize()
    assert torch.equal(out, want)


def test_two_streams_at_once(gpu):
    """Calls on two streams with workspaces and outputs of their own do not meet."""
    import torch
    g = np.random.default_rng(64)
    p = tlq.params(act_bits=8)
    c = Pool(g, gpu, [3000, 100], [1, 1], 2, 128, 64, "f16")
    b, cache = c.load()
    x, f, wc, ws = _linear_case(g, 40, 2056, 9001, "f16", 8)
    X, W, S, F = dev(x, gpu, "f16"), _padded(wc, gpu), dev(ws, gpu), dev(f, gpu)
    q = dev(rnd(g.standard_normal((2, 8 * 128)), "f16"), gpu, "f16")
    y0 = tlq.linear_i8(X, W, S, p, torch.empty((40, 9008), dtype=torch.float16, device=gpu)[:, :9001], factor=F).clone()
    a0 = tlq.kv_attention(q, 8, b, cache, p, torch.empty_like(q)).clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            y = torch.empty((40, 9008), dtype=torch.float16, device=gpu)[:, :9001]
            outs.append((tlq.linear_i8(X, W, S, p, y, factor=F), tlq.kv_attention(q, 8, b, cache, p, torch.empty_like(q))))
    torch.cuda.synchronize()
    for y, a in outs:
        assert torch.equal(y, y0) and torch.equal(a, a0)


def test_single_rows_of_any_stride(gpu):
    """The stride of a matrix of one row is never used."""
    import torch
    g = np.random.default_rng(65)
    p = tlq.params(act_bits=8)
    x, f, wc, ws = _linear_case(g, 1, 256, 24, "f16", 8)
    X = dev(x, gpu, "f16")
    column = X.reshape(256, 1).t()                            # [1, 256] with strides of one
    W, S = _padded(wc, gpu), dev(ws, gpu)
    a, b = (tlq.linear_i8(t, W, S, p, torch.empty((1, 24), dtype=torch.float16, device=gpu)) for t in (X, column))
    assert column.stride() == (1, 1) and torch.equal(a, b)
