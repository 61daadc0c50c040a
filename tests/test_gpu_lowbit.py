"""The block's other low-bit calls on the GPU against the 64-bit oracle: residual, norm and codes; products of codes with an epilogue;
rotation by positions on several axes; the 4-bit cache written, read and attended to; a run of them together, captured
graphs, streams."""
import numpy as np
import pytest

from oracle import lowbit as lo
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
    return a if dt == "f32" else lo.round16(a, dt == "bf16")


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


def untouched(wide, left, width):
    import torch
    keep = torch.ones(wide.shape[1], dtype=torch.bool, device=wide.device)
    keep[left:left + width] = False
    return bool((wide[:, keep] == 3.0).all())


def within(got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) / bound)), np.argwhere(bad)[:4].tolist())


def _kernels(call):
    """Names of the library's launches of a call."""
    tlq.profile_reset()
    tlq.profile_enable(True)
    try:
        call()
        return {k.name for k in tlq.profile_read() if k.launches}
    finally:
        tlq.profile_enable(False)
        tlq.profile_reset()


# ------------------------------------------------------------------ residual, norm, codes
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,c,bits,add,weight", [
    (1, 8, 8, True, False), (3, 72, 8, False, True), (17, 128, 4, True, True), (9, 1096, 2, True, False), (130, 520, 6, False, False),
    (5, 1024, 8, True, True), (4, 1032, 8, True, True), (2, 13824, 8, True, True), (5, 4104, 8, True, True), (3, 4096, 8, False, True),
    (2, 8200, 5, True, True), (3, 16392, 8, True, True), (2, 65536, 8, True, True), (1, 16384, 7, False, True), (301, 640, 8, True, True)])
def test_add_norm_codes_are_exact(gpu, dt, n, c, bits, add, weight):
    """h, codes and steps are those of the definition, bit for bit."""
    import torch
    g = np.random.default_rng([71, n, c])
    h = rnd(g.standard_normal((n, c)) * np.exp(2 * g.standard_normal((n, 1))), dt)
    h[:, g.integers(0, c, max(1, c // 50))] *= 32
    h = rnd(h, dt)
    z = rnd(g.standard_normal((n, c)), dt) if add else None
    if n > 2:
        h[0] = 0.0                                            # a row of zeros: eps alone
        if add:
            z[0] = 0.0
    w = np.exp(0.5 * g.standard_normal(c)).astype(np.float32) if weight else None
    c8 = -(-c // 128) * 128
    wide = torch.full((n, c8 + 32), 77, dtype=torch.int8, device=gpu)
    steps = torch.empty(n, device=gpu)
    H, Hw = spread(h, gpu, dt)
    Z = spread(z, gpu, dt)[0] if add else None
    out, outw = spread(np.zeros_like(h), gpu, dt)
    p = tlq.params(x_dtype=CODE[dt])
    call = lambda H_out: tlq.add_norm_codes(H, None if w is None else dev(w, gpu), p, wide[:, 16:16 + c8], steps, Z=Z, H_out=H_out, eps=1e-5, bits=bits)
    want = lo.add_norm_codes(h, z, w, 1e-5, bits, dt == "bf16")
    for H_out in (out, None, H):                              # (the last: in place)
        wide.fill_(77)
        steps.fill_(0)
        call(H_out)
        got = wide.cpu().numpy()
        assert np.array_equal(got[:, 16:16 + c], want[1]) and np.array_equal(steps.cpu().numpy(), want[2])
        assert np.all(got[:, 16 + c:16 + c8] == 0) and np.all(got[:, :16] == 77) and np.all(got[:, 16 + c8:] == 77)
        if H_out is not None:
            assert np.array_equal(host(H_out), want[0])
    assert untouched(outw, 8, c) and untouched(Hw, 8, c)


def test_add_norm_codes_are_those_of_the_calls_apart(gpu):
    """The residual's sum is tlq_residual_add's; codes of what is normalised already are tlq_row_codes'."""
    import torch
    g = np.random.default_rng(72)
    n, c, p = 40, 648, tlq.params(x_dtype=tlq.BF16)
    H, Z = (dev(rnd(g.standard_normal((n, c)), "bf16"), gpu, "bf16") for _ in range(2))
    new = lambda: (torch.empty((n, 768), dtype=torch.int8, device=gpu), torch.empty(n, device=gpu))
    (codes, steps), out = new(), torch.empty_like(H)
    tlq.add_norm_codes(H, None, p, codes, steps, Z=Z, H_out=out)
    assert torch.equal(out, tlq.residual_add(H, Z, p, torch.empty_like(H)))
    # rows of signs: normalised by one exactly, with eps = 0
    S = torch.sign(H.float()).to(torch.bfloat16)
    S[S == 0] = 1.0
    f = dev(np.exp(g.standard_normal(c)).astype(np.float32), gpu)
    (a, sa), (b, sb) = new(), new()
    tlq.add_norm_codes(S, f, p, a, sa, eps=0.0)
    tlq.row_codes(S, 8, p, b, sb, factor=f)
    assert torch.equal(a, b) and torch.equal(sa, sb)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,c", [(5, 136), (3, 1096), (3, 5120), (2, 13824), (2, 20008), (2, 40008)])
def test_add_norm_codes_onto_the_second_matrix(gpu, dt, n, c):
    """H_out may be Z; H and Z may be the same."""
    import torch
    g = np.random.default_rng([103, n, c])
    h, z = (rnd(g.standard_normal((n, c)), dt) for _ in range(2))
    H, Z = dev(h, gpu, dt), dev(z, gpu, dt)
    codes, steps = torch.empty((n, -(-c // 128) * 128), dtype=torch.int8, device=gpu), torch.empty(n, device=gpu)
    p = tlq.params(x_dtype=CODE[dt])
    for a, b, second in ((H, Z, z), (H, H, h)):
        tlq.add_norm_codes(a, None, p, codes, steps, Z=b, H_out=b, eps=1e-5)
        want = lo.add_norm_codes(h, second, None, 1e-5, 8, dt == "bf16")
        assert np.array_equal(host(b), want[0]) and np.array_equal(codes.cpu().numpy()[:, :c], want[1]) and np.array_equal(steps.cpu().numpy(), want[2])


@pytest.mark.parametrize("dt,c", [("f16", 264), ("bf16", 5120)])
def test_add_norm_codes_of_rows_that_are_not_finite(gpu, dt, c):
    """Such a row has a NaN step, and its products are NaN; the others do not see it.  Zeros without eps likewise."""
    import torch
    g = np.random.default_rng(73)
    h = rnd(g.standard_normal((6, c)), dt)
    z = np.zeros_like(h)
    h[1, 5], h[2, c - 1], h[4] = np.inf, np.nan, 0.0
    h[3, 7] = z[3, 7] = 60000.0 if dt == "f16" else 3e38      # (the sum is an infinity)
    h[3], z[3] = rnd(h[3], dt), rnd(z[3], dt)
    p = tlq.params(x_dtype=CODE[dt])
    c8 = -(-c // 128) * 128
    codes, steps = torch.empty((6, c8), dtype=torch.int8, device=gpu), torch.empty(6, device=gpu)
    tlq.add_norm_codes(dev(h, gpu, dt), None, p, codes, steps, Z=dev(z, gpu, dt), eps=0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        want = lo.add_norm_codes(h[[0, 5]], z[[0, 5]], None, 0.0, 8, dt == "bf16")
    s = steps.cpu().numpy()
    assert np.isnan(s[1:5]).all() and np.array_equal(s[[0, 5]], want[2]) and np.array_equal(codes.cpu().numpy()[[0, 5], :c], want[1])
    y = tlq.linear_codes(codes, steps, c, torch.ones((5, c8), dtype=torch.int8, device=gpu), torch.ones(5, device=gpu), p,
                         torch.empty((6, 8), dtype=torch.float16, device=gpu)[:, :5])
    assert bool(y[1:5].isnan().all()) and bool(y[[0, 5]].isfinite().all())


def test_add_norm_codes_of_squares_beyond_floats(gpu):
    """bf16 rows near the type's largest and smallest numbers."""
    import torch
    g = np.random.default_rng(74)
    h = rnd(g.standard_normal((8, 520)) * 2.0 ** np.array([120, 90, 64, 0, -50, -64, -100, -126])[:, None], "bf16")
    codes, steps = torch.empty((8, 640), dtype=torch.int8, device=gpu), torch.empty(8, device=gpu)
    tlq.add_norm_codes(dev(h, gpu, "bf16"), None, tlq.params(x_dtype=tlq.BF16), codes, steps, eps=0.0)
    want = lo.add_norm_codes(h, None, None, 0.0, 8, True)
    assert np.array_equal(codes.cpu().numpy()[:, :520], want[1]) and np.array_equal(steps.cpu().numpy(), want[2])


# ------------------------------------------------------------------ products of codes with an epilogue
def _linear_case(g, n, ci, co, bits=8):
    top = 2 ** (bits - 1) - 1
    codes, w = g.integers(-top, top + 1, (n, ci)).astype(np.int8), g.integers(-127, 128, (co, ci)).astype(np.int8)
    steps = np.exp(0.3 * g.standard_normal(n)).astype(np.float32) / top
    ws = (np.exp(0.3 * g.standard_normal(co)) / (127 * np.sqrt(ci) / 1.5)).astype(np.float32)
    return codes, steps, w, ws


def _padded(c, gpu, extra=0):
    import torch
    n, ci = c.shape
    t = torch.zeros((n, -(-ci // 128) * 128 + extra), dtype=torch.int8, device=gpu)
    if extra:
        t[:, -extra:] = 99
    t[:, :ci] = dev(c, gpu)
    return t


def _linear_bound(p, v, a, y, kind, r, mul, od, x=None):
    """The sum as a float and its two products (3 roundings), the bias (1); the activation's derivative is 1.13 at most.  Its own error:
    logistic, an exponential whose argument x is off by 4 roundings of itself (two constants, a product, a sum with one of equal
    sign, a product) and 8 further ones; normal distribution, 20, and 3 of v^2 / 2 (a constant, two products), in the tail that
    is taken from v above zero; what is below 1e-36 may be zero; the second matrix (1); the output."""
    dv = np.abs(p) * 3.1 * U + np.abs(v) * 1.1 * U
    x = v if x is None else x
    if kind == 0:
        da = dv
    elif kind == 3:
        tail = np.where(x >= 0, np.abs(x - a), np.abs(a))
        da = 1.13 * dv + (tail * (20 + 1.5 * np.minimum(x * x, 1e4)) + np.abs(a)) * U + 1e-36
    else:
        arg = np.minimum(np.abs(x if kind == 1 else 1.6 * (x + 0.0447 * np.clip(x, -1e3, 1e3) ** 3)), 1e4)
        tail = np.where(x >= 0, np.abs(x - a), np.abs(a))
        da = 1.13 * dv + (tail * 4 * arg + np.abs(a) * 8) * U + 1e-36
    if r is not None:
        da = (da * np.abs(r) if mul else da) + np.abs(y) * U
    return da * 1.01 + (np.abs(y) + da) * HALF[od] + TINY[od] * 1.01


FEW, MID, ONE, TILES, STORE = {"linear_few"}, {"linear_mid", "linear_join"}, {"linear_mid"}, {"gemm_finish"}, {"gemm_store"}
EPILOGUES = [(1, 3, "mul"), (1, 0, "add"), (0, 1, "mul"), (1, 2, ""), (0, 3, ""), (0, 0, "add"), (1, 1, "add")]


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,ci,co,kernels", [
    (1, 8, 1, FEW), (1, 4096, 16, FEW), (2, 72, 3, FEW), (17, 136, 31, FEW), (33, 2056, 50, FEW), (64, 384, 130, FEW), (300, 1096, 263, FEW),
    (16, 8200, 9001, MID), (40, 8200, 8001, MID), (64, 8200, 2203, MID), (200, 4104, 1003, MID), (33, 512, 70001, ONE),
    # tiles of 128 outputs x 64 tokens, where they are one a CU at most; of 128 x 128, as many and more; of 256 outputs x 192,
    # 256 and 320 tokens; ragged and whole
    (1, 136, 20481, TILES), (16, 264, 32768, TILES), (40, 2568, 13000, TILES), (64, 128, 8192, TILES), (130, 2184, 3401, TILES), (300, 4104, 263, TILES),
    (1152, 256, 2048, TILES), (1000, 264, 2051, TILES), (1024, 256, 2048, TILES), (2501, 136, 2050, TILES), (6391, 136, 2557, TILES),
    (2496, 128, 4096, TILES), (4001, 136, 2051, TILES), (4000, 128, 4002, TILES), (4096, 128, 4096, TILES), (4800, 128, 4096, TILES), (8001, 136, 2051, TILES)])
def test_linear_codes(gpu, out, n, ci, co, kernels):
    """Every kernel of the product, each named, with every activation, a bias, a second matrix added and multiplied."""
    import torch
    g = np.random.default_rng([75, n, ci, co])
    codes, steps, w, ws = _linear_case(g, n, ci, co)
    bias, r = g.standard_normal(co).astype(np.float32), rnd(g.standard_normal((n, co)), out)
    p = tlq.params(yref_dtype=CODE[out])
    X, S, W, WS, B = _padded(codes, gpu, 16), dev(steps, gpu), _padded(w, gpu, 32), dev(ws, gpu), dev(bias, gpu)
    R, _ = spread(r, gpu, out)
    work = torch.full((max(256, tlq.linear_codes_workspace_bytes(n, ci)),), 0xAB, dtype=torch.uint8, device=gpu)
    # (the product in 64 bits once; three epilogues of the seven a shape, another three a type)
    plain, product, _, _ = lo.linear_codes(codes, steps, w, ws, None, 0, None, False)
    first = (n + 3 * ["f16", "bf16", "f32"].index(out)) % len(EPILOGUES)
    for k in range(3 if n * co > 1 << 20 else len(EPILOGUES)):
        b, kind, second = EPILOGUES[(first + k) % len(EPILOGUES)]
        y, wide = spread(np.zeros((n, co), np.float32), gpu, out)
        y.fill_(9.0)
        call = lambda: tlq.linear_codes(X, S, ci, W, WS, p, y, bias=B if b else None, act=kind, R=R if second else None, mul=second == "mul", workspace=work)
        assert _kernels(call) == kernels
        v = product + bias.astype(np.float64) if b else product
        a = lo.act(v, kind)
        want = a + r if second == "add" else a * r if second == "mul" else a
        within(host(y), want, _linear_bound(product, v, a, want, kind, r if second else None, second == "mul", out))
        assert untouched(wide, 8, co)


@pytest.mark.parametrize("n,ci,co", [(5, 640, 70), (40, 2568, 13000), (300, 4104, 263), (2501, 136, 2050)])
def test_linear_codes_without_an_epilogue_is_linear_i8(gpu, n, ci, co):
    import torch
    g = np.random.default_rng([76, n])
    x = rnd(g.standard_normal((n, ci)), "bf16")
    p = tlq.params(act_bits=8, x_dtype=tlq.BF16, yref_dtype=tlq.BF16)
    X = dev(x, gpu, "bf16")
    codes, steps = torch.empty((n, -(-ci // 128) * 128), dtype=torch.int8, device=gpu), torch.empty(n, device=gpu)
    tlq.row_codes(X, 8, p, codes, steps)
    _, _, w, ws = _linear_case(g, 1, ci, co)
    W, WS = _padded(w, gpu), dev(ws, gpu)
    a, b = (torch.empty((n, -(-co // 8) * 8), dtype=torch.bfloat16, device=gpu)[:, :co] for _ in range(2))
    tlq.linear_i8(X, W, WS, p, a)
    tlq.linear_codes(codes, steps, ci, W, WS, p, b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("n,co", [(3, 40), (64, 2203), (300, 263), (1100, 2048), (4096, 4096)])
@pytest.mark.parametrize("mul", [False, True])
def test_linear_codes_onto_its_second_matrix(gpu, n, co, mul):
    """Y may be R: the residual stream is updated in place."""
    import torch
    g = np.random.default_rng([77, n])
    ci = 8200 if n == 64 else 264
    codes, steps, w, ws = _linear_case(g, n, ci, co)
    X, S, W, WS, p = _padded(codes, gpu), dev(steps, gpu), _padded(w, gpu), dev(ws, gpu), tlq.params()
    R = torch.empty((n, -(-co // 8) * 8), dtype=torch.float16, device=gpu)[:, :co]
    R.copy_(dev(rnd(g.standard_normal((n, co)), "f16"), gpu, "f16"))
    y = torch.empty((n, -(-co // 8) * 8), dtype=torch.float16, device=gpu)[:, :co]
    tlq.linear_codes(X, S, ci, W, WS, p, y, act=tlq.ACT_SILU, R=R, mul=mul)
    tlq.linear_codes(X, S, ci, W, WS, p, R, act=tlq.ACT_SILU, R=R, mul=mul)
    assert torch.equal(R, y)


@pytest.mark.parametrize("kind", [1, 2, 3])
@pytest.mark.parametrize("n", [1, 300])
def test_activations_over_their_range(gpu, kind, n):
    """One value an output, from where the activation is the value to where it is nothing, exactly representable ones: the error is
    the activation's own.  Few tokens and tiles."""
    g = np.random.default_rng(78)
    v = np.concatenate([np.linspace(-14, 14, 3001), -np.exp(np.linspace(-30, 8, 500)), np.exp(np.linspace(-30, 8, 500)), [0.0, 1e30, -1e30, 3e38, -3e38]]).astype(np.float32)
    co = len(v)
    ci = 8 if n == 1 else 2176
    codes = np.zeros((n, ci), np.int8)
    w = np.zeros((co, ci), np.int8)
    codes[:, 0], w[:, 0] = 1, 1
    import torch
    y = torch.empty((n, -(-co // 4) * 4), device=gpu)[:, :co]
    tlq.linear_codes(_padded(codes, gpu), dev(np.ones(n, np.float32), gpu), ci, _padded(w, gpu), dev(v, gpu), tlq.params(yref_dtype=tlq.F32), y, act=kind)
    v = v.astype(np.float64)
    a = lo.act(v, kind)
    within(host(y), np.broadcast_to(a, (n, co)), _linear_bound(0 * v, 0 * v, a, a, kind, None, False, "f32", v))


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
@pytest.mark.parametrize("n,ci,co", [(3, 264, 50), (40, 2568, 13000), (64, 8200, 2203), (300, 4104, 263), (2501, 136, 2050)])
def test_linear_codes_of_numbers_that_are_not_finite(gpu, kind, n, ci, co):
    """Infinities and NaN in a bias, a row whose step is NaN (as the norm marks it): they stay in their outputs and rows."""
    import torch
    g = np.random.default_rng([79, n])
    codes, steps, w, ws = _linear_case(g, n, ci, co)
    bias = g.standard_normal(co).astype(np.float32)
    X, W, WS, p = _padded(codes, gpu), _padded(w, gpu), dev(ws, gpu), tlq.params()
    clean, odd = (torch.empty((n, -(-co // 8) * 8), dtype=torch.float16, device=gpu)[:, :co] for _ in range(2))
    tlq.linear_codes(X, dev(steps, gpu), ci, W, WS, p, clean, bias=dev(bias, gpu), act=kind)
    steps[n // 2], bias[5], bias[co - 1], bias[17] = np.nan, np.inf, np.nan, -np.inf
    tlq.linear_codes(X, dev(steps, gpu), ci, W, WS, p, odd, bias=dev(bias, gpu), act=kind)
    rest = torch.ones((n, co), dtype=torch.bool, device=gpu)
    rest[n // 2] = rest[:, 5] = rest[:, co - 1] = rest[:, 17] = False
    assert torch.equal(odd[rest], clean[rest])
    assert bool(odd[n // 2].isnan().all()) and bool(odd[:, co - 1].isnan().all())
    there = [t for t in range(n) if t != n // 2]
    assert bool((odd[there, 5] == float("inf")).all())
    low = odd[there, 17]
    assert bool({0: low == float("-inf"), 3: low == 0}.get(kind, low.isnan()).all())


def test_linear_codes_extreme_sums(gpu):
    """The largest sums that the codes allow, 2^30, with a bias that nearly cancels them."""
    import torch
    ci, co = 65536, 5
    for rows in (2, 66, 300):
        codes = torch.full((rows, ci), 127, dtype=torch.int8, device=gpu)
        codes[1::2] = -128
        w = torch.full((co, ci), -128, dtype=torch.int8, device=gpu)
        y = torch.empty((rows, 8), device=gpu)[:, :co]
        bias = torch.full((co,), float(127 * 128 * ci), device=gpu)
        tlq.linear_codes(codes, torch.ones(rows, device=gpu), ci, w, torch.ones(co, device=gpu), tlq.params(yref_dtype=tlq.F32), y, bias=bias)
        want = np.where(np.arange(rows) % 2 == 0, -127.0 * 128 * ci, 128.0 * 128 * ci)[:, None] + 127.0 * 128 * ci
        within(host(y), np.broadcast_to(want, (rows, co)), 2.0 ** 30 * 4 * U)


# ------------------------------------------------------------------ positions on several axes
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,h,kv,dh,rot,pairs,norm,far,axes", [
    (1, 1, 1, 64, 64, False, True, 10, 3), (5, 3, 1, 128, 128, False, True, 5000, 3), (16, 32, 8, 128, 128, False, True, 2 ** 31 - 1, 2),
    (7, 7, 1, 128, 64, False, False, 1000, 4), (33, 5, 5, 256, 256, True, True, 100000, 3), (4, 2, 2, 64, 48, False, True, 77, 1),
    (9, 4, 2, 64, 16, True, False, 3000, 3), (6, 2, 1, 128, 0, False, True, 9, 3), (8200, 1, 1, 64, 64, False, True, 9000, 3)])
def test_qk_norm_rope_axes(gpu, dt, n, h, kv, dh, rot, pairs, norm, far, axes):
    import torch
    g = np.random.default_rng([79, n, h, dh, rot])
    q, k = (rnd(g.standard_normal((n, m * dh)) * np.exp(g.standard_normal((n, 1))), dt) for m in (h, kv))
    q[0] = 0.0
    pos = g.integers(0, far, (axes, n)).astype(np.int32)
    pos[-1, -1] = -(2 ** 31)
    axis = (np.arange(rot // 2) % (axes + 1) if pairs else np.arange(rot // 2) * axes // max(1, rot // 2)).astype(np.int32)
    if len(axis):
        axis[0], axis[-1] = -7, 2 ** 31 - 1                    # (held to the axes that there are)
    inv = 1e6 ** (-np.arange(rot // 2) / max(1, rot // 2))
    w = [np.exp(0.3 * g.standard_normal(dh)).astype(np.float32) if norm else None for _ in range(2)]
    p = tlq.params(x_dtype=CODE[dt])
    both, _ = spread(np.concatenate([q, k], 1), gpu, dt)
    qo, qw = spread(np.zeros_like(q), gpu, dt)
    ko, kw = spread(np.zeros_like(k), gpu, dt)
    wide_pos = torch.full((axes, n + 3), 12345, dtype=torch.int32, device=gpu)
    wide_pos[:, :n] = dev(pos, gpu)
    args = (dh, wide_pos[:, :n], dev(axis, gpu) if rot else None, dev(inv, gpu) if rot else None, p)
    kw_args = dict(wq=None if w[0] is None else dev(w[0], gpu), wk=None if w[1] is None else dev(w[1], gpu), norm=norm, interleaved=pairs)
    tlq.qk_norm_rope_axes(both[:, :h * dh], both[:, h * dh:], *args, qo, ko, **kw_args)
    top = np.abs(pos.astype(np.float64)).max(axis=0)[:, None, None]
    for x, got, wt in ((q, qo, w[0]), (k, ko, w[1])):
        want = lo.norm_rope_axes(x, dh, pos, axis, inv, wt, 1e-6, norm, pairs)
        u = np.abs(lo.norm_rope_axes(x, dh, pos, axis[:0], inv[:0], wt, 1e-6, norm, pairs)).reshape(n, -1, dh)
        pair = u.copy()                                       # |u_a| + |u_b| of each pair
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            pair[:, :, a] = pair[:, :, b] = u[:, :, a] + u[:, :, b]
        # the norm: dh products summed in any order, a root, a quotient, two products; cosine and sine: a fraction of a turn
        # as a float (2 pi 2^-26), the function's own error (two ulp of 1), the angle in double
        delta = (dh + 8) * U + 2 * np.pi * 2.0 ** -26 + 4 * U + top * 2.0 ** -51
        within(host(got).reshape(n, -1, dh), want.reshape(n, -1, dh), pair * delta + np.abs(want).reshape(n, -1, dh) * HALF[dt] * 1.001 + TINY[dt] * 1.01)
    assert untouched(qw, 8, h * dh) and untouched(kw, 8, kv * dh)
    # where a token's positions agree: the bits of one axis
    args[1][:] = args[1][0].clone()
    tlq.qk_norm_rope_axes(both[:, :h * dh], both[:, h * dh:], *args, qo, ko, **kw_args)
    qo1, ko1 = torch.empty_like(qo), torch.empty_like(ko)
    tlq.qk_norm_rope(both[:, :h * dh], both[:, h * dh:], dh, args[1][0], args[3], p, qo1, ko1, **kw_args)
    assert torch.equal(qo, qo1) and torch.equal(ko, ko1)
    # in place
    tlq.qk_norm_rope_axes(both[:, :h * dh], both[:, h * dh:], *args, both[:, :h * dh], both[:, h * dh:], **kw_args)
    assert torch.equal(both[:, :h * dh], qo) and torch.equal(both[:, h * dh:], ko)


# ------------------------------------------------------------------ the cache
class Pool:
    """Pages of several sequences in no order, codes and steps as the oracle has them, and their copies on the GPU."""

    def __init__(self, g, gpu, lens, new, kv, dh, page, dt, spare=2):
        self.gpu, self.dt = gpu, dt
        self.new, self.lens, self.kv, self.dh, self.page = list(new), list(lens), kv, dh, page
        need = [-(-max(n, 0) // page) for n in lens]
        self.n = sum(need) + spare
        order = g.permutation(self.n)
        self.table = np.full((len(lens), max(max(need), 1) + 1), -1, np.int32)
        at = 0
        for s, m in enumerate(need):
            self.table[s, :m] = order[at:at + m]
            at += m
        self.kc = g.integers(-8, 8, (self.n, kv, page, dh)).astype(np.int8)
        self.vc = g.integers(-8, 8, (self.n, kv, dh, page)).astype(np.int8)
        step = lambda *sh: rnd(0.15 * np.exp(0.5 * g.standard_normal(sh)), "bf16").astype(np.float16)
        self.ks, self.vs = step(self.n, kv, page, dh // 32), step(self.n, kv, dh // 32, page)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.rows = int(self.cu[-1])
        self.max_new, self.max_len = max(max(new), 1), max(max(lens), max(new), 1)

    def load(self):
        d = lambda a: dev(a, self.gpu)
        self.t = (d(lo.pack(self.kc)), d(self.ks), d(lo.pack(self.vc)), d(self.vs))
        self.l = np.array(self.lens, np.int32)
        return tlq.kv_batch(d(self.cu), d(self.l), d(self.table), self.max_new, self.max_len), tlq.kv4_cache(*self.t)

    def append(self, x, y, max_new=None):
        lo.kv4_append(x, self.kc, self.ks, self.cu, self.lens, self.table, self.max_len, False, max_new)
        lo.kv4_append(y, self.vc, self.vs, self.cu, self.lens, self.table, self.max_len, True, max_new)

    def held(self):
        """Whether the GPU's cache is the oracle's, bit for bit."""
        k, ks, v, vs = (t.cpu().numpy() for t in self.t)
        return (np.array_equal(k, lo.pack(self.kc)) and np.array_equal(v, lo.pack(self.vc)) and
                np.array_equal(ks.view(np.uint16), self.ks.view(np.uint16)) and np.array_equal(vs.view(np.uint16), self.vs.view(np.uint16)))

    def values(self):
        with np.errstate(invalid="ignore"):
            return lo.values(self.kc, self.ks, False), lo.values(self.vc, self.vs, True)


APPENDS = [
    ([1], [1], 1, 64, 16), ([16, 17, 33], [16, 1, 33], 2, 128, 16), ([100, 64, 65, 1], [37, 64, 1, 1], 3, 128, 64),
    ([200, 0, 5], [90, 0, 5], 2, 64, 128), ([300, 299], [3, 299], 1, 128, 256), ([48, 40, 47], [9, 40, 2], 5, 128, 32),
    ([2, 130], [5, 2], 2, 64, 32),           # more new rows than the sequence has tokens
    ([300, 128, 129, 1], [190, 100, 129, 1], 2, 128, 128), ([700, 256, 257, 300], [500, 130, 257, 299], 3, 64, 256),
    ([7, 8, 9, 15, 16], [7, 8, 9, 8, 7], 1, 64, 16), ([70, 17], [60, 16], 40, 128, 16), ([9, 9, 9], [1, 2, 8], 7, 64, 64),
]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,kv,dh,page", APPENDS)
def test_kv4_append_and_read(gpu, dt, lens, new, kv, dh, page):
    """Words and steps are those of the definition, bit for bit; what is not written stays as it was; and back again."""
    import torch
    g = np.random.default_rng([81, sum(lens), page, dh])
    c = Pool(g, gpu, lens, new, kv, dh, page, dt)
    rows = c.rows + 3                                         # rows behind the last sequence: no part in anything
    x = rnd(g.standard_normal((rows, 2 * kv * dh)) * np.exp(1.5 * g.standard_normal((rows, 1))), dt)
    x[c.rows:] = np.nan
    x[0, :dh] = 0.0
    b, cache = c.load()
    p = tlq.params(x_dtype=CODE[dt])
    wide, _ = spread(x, gpu, dt)
    tlq.kv4_append(wide[:, :kv * dh], wide[:, kv * dh:], b, cache, p)
    c.append(x[:, :kv * dh], x[:, kv * dh:])
    assert c.held()
    (ko, kw), (vo, vw) = (spread(np.zeros((rows, kv * dh), np.float32), gpu, dt) for _ in range(2))
    kw.fill_(3.0)
    vw.fill_(3.0)
    tlq.kv4_read(b, cache, p, ko, vo)
    for got, wd, (codes, steps, turned) in ((ko, kw, (c.kc, c.ks, False)), (vo, vw, (c.vc, c.vs, True))):
        want = lo.kv4_read(codes, steps, c.cu, c.lens, c.table, rows, c.max_len, turned)
        assert np.array_equal(host(got)[:c.rows], rnd(want[:c.rows], dt)) and (host(got)[c.rows:] == 3.0).all() and untouched(wd, 8, kv * dh)
    # one of them alone; the whole of the sequences, old tokens among them
    for name, got in (("K_out", ko), ("V_out", vo)):
        alone = torch.full_like(got, 3.0)
        tlq.kv4_read(b, cache, p, **{name: alone})
        assert torch.equal(alone, got)
    whole = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    every = tlq.kv_batch(dev(whole, gpu), b.parts[1], b.parts[2], max(max(lens), 1), c.max_len)
    ko, vo = (torch.empty((int(whole[-1]), kv * dh), dtype=tt(dt), device=gpu) for _ in range(2))
    tlq.kv4_read(every, cache, p, ko, vo)
    for got, (codes, steps, turned) in ((ko, (c.kc, c.ks, False)), (vo, (c.vc, c.vs, True))):
        assert np.array_equal(host(got), rnd(lo.kv4_read(codes, steps, whole, lens, c.table, int(whole[-1]), c.max_len, turned), dt))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_kv4_append_of_every_number(gpu, dt):
    """All 65,536 numbers of the type beside maxima of every size: infinities, NaN, subnormals, ties."""
    import torch
    g = np.random.default_rng(82)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(tt(dt)).float().numpy()
    x = np.concatenate([np.sort(np.abs(x)), x[g.permutation(65536)]]).reshape(2048, 64)      # (groups of like sizes, and of all)
    c = Pool(g, gpu, [2048], [2048], 1, 64, 256, dt)
    b, cache = c.load()
    X = dev(x, gpu, dt)
    tlq.kv4_append(X, X, b, cache, tlq.params(x_dtype=CODE[dt]))
    c.append(x, x)
    assert c.held()


def test_kv4_append_ties(gpu):
    """Values half way between two codes, for steps of every significand."""
    g = np.random.default_rng(83)
    m = np.arange(128, 256, dtype=np.float32) / 128           # significands of a step: 7 m is a half, the largest value
    x = np.zeros((256, 64), np.float32)
    for i, s in enumerate(m):
        for k, e in enumerate((0, -9)):
            row = np.concatenate([[7.0], np.arange(-6, 7) + 0.5, np.arange(-7, 8), np.zeros(3)]) * s * 2.0 ** e
            x[2 * i + k, :32], x[2 * i + k, 32:] = row, -row
    x = rnd(x, "f16")                                         # (odd significands times 9, 11 and 13 have twelve bits)
    c = Pool(g, gpu, [256], [256], 1, 64, 32, "f16")
    b, cache = c.load()
    tlq.kv4_append(dev(x, gpu, "f16"), dev(x, gpu, "f16"), b, cache, tlq.params())
    c.append(x, x)
    assert c.held()


@pytest.mark.parametrize("page", [16, 64])
def test_kv4_codes_do_not_hang_on_how_tokens_are_dealt(gpu, page):
    """One by one, in odd pieces and at once: the same cache."""
    import torch
    g = np.random.default_rng(84)
    kv, dh, n = 2, 128, 61
    c = Pool(g, gpu, [n], [n], kv, dh, page, "bf16")
    x = rnd(g.standard_normal((n, kv * dh)) * np.exp(g.standard_normal((n, 1))), "bf16")
    X = dev(x, gpu, "bf16")
    p = tlq.params(x_dtype=tlq.BF16)
    b, cache = c.load()
    start = [t.clone() for t in c.t]
    tlq.kv4_append(X, X, b, cache, p)
    want = [t.clone() for t in c.t]
    for deal in ([1] * n, [5, 1, 13, 3, 8, 16, 2, 13]):
        for t, o in zip(c.t, start):
            t.copy_(o)
        at = 0
        for m in deal:
            part = tlq.kv_batch(dev(np.array([0, m], np.int32), gpu), dev(np.array([at + m], np.int32), gpu), b.parts[2], m, n)
            tlq.kv4_append(X[at:at + m], X[at:at + m], part, cache, p)
            at += m
        assert at == n and all(torch.equal(t, o) for t, o in zip(c.t, want))


def _attend(gpu, c, heads, dt, q, scale=0.0):
    import torch
    b, cache = c.load()
    wide_q, _ = spread(q, gpu, dt)
    out, wide = spread(np.zeros_like(q), gpu, dt)
    wide.fill_(3.0)
    p = tlq.params(x_dtype=CODE[dt])
    work = torch.full((max(256, tlq.kv4_attention_workspace_bytes(q.shape[0], heads, b, cache)),), 0xFF, dtype=torch.uint8, device=gpu)
    tlq.kv4_attention(wide_q, heads, b, cache, p, out, scale=scale, workspace=work)
    torch.cuda.synchronize()
    assert untouched(wide, 8, q.shape[1])
    return host(out)


def _bounds(c, heads, q, kind):
    """Host's bounds under which the tiles of 128 rows are taken (they need work for many blocks): rows behind the last sequence
    ("tiles"), or, for more than 48 rows, longer sequences than there are ("parts": many parts, most of them empty)."""
    group, pairs = heads // c.kv, len(c.lens) * c.kv
    if kind == "tiles":
        q = np.concatenate([q, np.full((3340 * 16 // (group * pairs) + 16, q.shape[1]), np.nan)])
        c.max_new = q.shape[0]
        c.max_len = max(c.max_len, c.max_new)
    if kind == "parts":
        units = 3340 // (max(-(-c.max_new * group // 16), 1) * pairs) + 1
        c.max_len = max(c.max_len, units * 256)
        c.table = np.concatenate([c.table, np.full((len(c.lens), max(0, -(-c.max_len // c.page) - c.table.shape[1])), -1, np.int32)], 1)
    return q


def _bound(c, dt, want, mag, sens, top):
    """Weights in 16 bits, above the line and below it: sum_j p_j e_j (v_j - out), |e_j| <= 2^-11, at most 2^-11 (mag + |out|); those below
    2^-21 of the largest to 2^-32 of it; scores as sums of dh products (a relative error of e^(2 ds) in p and in the sum of p), sums
    over the keys in 32 bits, the output.  `top`: the largest value."""
    n = min(c.max_len, max(c.lens))
    ds = ((c.dh + 6) * np.repeat(sens, c.dh, 1) + 64) * U
    return ((mag + np.abs(want)) * 2.0 ** -11 + mag * (2.1 * ds + (n / 4 + 64) * U) + n * 2.0 ** -32 * (top + np.abs(want)) +
            np.abs(want) * HALF[dt] * 1.001 + TINY[dt] * 1.01)


def _check_attention(gpu, c, heads, dt, q, scale=0.0):
    got = _attend(gpu, c, heads, dt, q, scale)
    k, v = c.values()
    want, mag, sens = lo.attention(q, heads, k, v, c.cu, c.lens, c.table, c.max_len, scale or None)
    none = np.isnan(mag[:, 0]) & ~(np.arange(len(q)) < c.rows)
    assert np.all(got[none] == 3.0)                            # rows behind the last sequence stay as they were
    got, want, mag, sens = got[~none], want[~none], mag[~none], sens[~none]
    bound = _bound(c, dt, want, mag, sens, np.nanmax(np.abs(v)))
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
def test_kv4_attention(gpu, dt, kind, lens, new, kv, group, dh, page):
    g = np.random.default_rng([85, sum(lens), group, dh])
    c = Pool(g, gpu, lens, new, kv, dh, page, dt)
    q = rnd(1.5 * g.standard_normal((c.rows + 2, kv * group * dh)), dt)
    q[c.rows:] = np.nan
    _check_attention(gpu, c, kv * group, dt, _bounds(c, kv * group, q, kind))


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("lens,new,kv,group,dh,page", ATTENTION)
def test_kv4_attention_runs_the_kernel_that_its_bounds_are_for(gpu, kind, lens, new, kv, group, dh, page):
    """Tiles of 16 rows by the batches' own bounds; by those of `_bounds` tiles of 128, for more than 48 rows where only the length grows."""
    g = np.random.default_rng(102)
    c = Pool(g, gpu, lens, new, kv, dh, page, "f16")
    q = _bounds(c, kv * group, np.zeros((c.rows, kv * group * dh), np.float32), kind)
    want = "kv4_prompt" if kind == "tiles" or (kind == "parts" and max(new) * group > 48) else "kv4_few"
    b, cache = c.load()
    Q = dev(np.nan_to_num(q), gpu, "f16")
    names = _kernels(lambda: tlq.kv4_attention(Q, kv * group, b, cache, tlq.params(), Q.clone()))
    assert want in names and names <= {want, "kv_join"}


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_kv4_attention_of_wild_steps_and_loud_queries(gpu, dt, kind):
    """Steps from the smallest to the largest, subnormal halves among them; queries of very different size, zeros among them; scores
    large enough that one key has nearly all of the weight; a scale of the caller's."""
    g = np.random.default_rng(86)
    c = Pool(g, gpu, [400, 333, 90], [1, 6, 90], 2, 128, 16, dt)
    c.vs[:] = np.minimum(rnd(1e-6 * np.exp(g.uniform(0, 23, c.vs.shape)), "bf16"), 9344.0).astype(np.float16)
    c.vc[:] = np.maximum(c.vc, -7)                             # (eight of the largest steps are no half, and no append writes them)
    q = rnd(g.standard_normal((c.rows, 4 * 128)) * np.exp(2 * g.standard_normal((c.rows, 1))), dt)
    q[2] = 0.0
    if dt == "bf16":
        q[3] = rnd(q[3] * 2.0 ** -100, dt)
    q = _bounds(c, 4, q, kind)
    if dt == "f16":                                            # (outputs up to the type's largest)
        c.vs[:] = np.minimum(c.vs, np.float16(4000.0))
    _check_attention(gpu, c, 4, dt, q)
    _check_attention(gpu, c, 4, dt, q, scale=-0.31)
    c.ks[:] = (c.ks.astype(np.float32) * 16).astype(np.float16)
    _check_attention(gpu, c, 4, dt, q)
    c.ks[:] = np.float16(2.0 ** -24)                           # (keys that are subnormal halves; a scale that makes up for them)
    _check_attention(gpu, c, 4, dt, q, scale=2.0 ** 18)


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("page,dh", [(16, 128), (16, 64), (32, 128), (256, 64)])
def test_kv4_attention_does_not_see_what_lies_behind_the_last_token(gpu, kind, dt, page, dh):
    """Steps and codes behind a sequence's last token in its page, in pages that the table names ahead, and in pages that are no
    page: they may hold anything."""
    g = np.random.default_rng([87, page, dh])
    lens, new = [33, 70, 17, 272, 300, 5], [33, 50, 1, 20, 16, 5]
    c = Pool(g, gpu, lens, new, 2, dh, page, dt, spare=8)
    c.table = np.concatenate([c.table, np.full((6, 4), -1, np.int32)], 1)
    if page < 64:
        c.table[3, 2], c.table[4, 0], c.table[1, 1] = -5, 2 ** 31 - 1, c.n
    c.table[5, :] = -1                                         # (a sequence without pages: zeros)
    spare = [i for i in range(c.n) if i not in set(c.table.ravel().tolist())]
    q = _bounds(c, 4, rnd(g.standard_normal((c.rows, 4 * dh)), dt), kind)
    want = _attend(gpu, c, 4, dt, q)[:c.rows]
    assert np.isfinite(want).all() and (want[-5:] == 0.0).all()
    ahead = spare[:4]
    for s, n in enumerate(lens[:5]):
        m = -(-n // page)
        c.table[s, m:][:3] = np.array(ahead)[[s % 4, (s + 1) % 4, 0]]
        last = int(c.table[s, m - 1])
        if 0 <= last < c.n and n % page:
            c.ks[last, :, n % page:], c.vs[last, :, :, n % page:] = np.nan, np.inf
            c.kc[last, :, n % page:], c.vc[last, :, :, n % page:] = 7, -8
    for k, v in ((np.nan, np.inf), (np.inf, np.nan), (0.0, -np.inf), (65504.0, 65504.0)):
        c.ks[spare], c.vs[spare] = np.float16(k), np.float16(v)
        assert np.array_equal(_attend(gpu, c, 4, dt, q)[:c.rows], want), (k, v)


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
def test_kv4_attention_of_pages_that_are_not_there(gpu, kind):
    """Entries outside the pool stand for tokens that do not exist, wherever they are; a row that sees none gives zeros."""
    g = np.random.default_rng(88)
    for dt, new in (("f16", [1, 3, 1, 2, 70]), ("bf16", [70, 40, 20, 30, 64])):
        c = Pool(g, gpu, [130, 100, 20, 40, 70], new, 2, 128, 16, dt)
        c.table[0, 2], c.table[0, 5], c.table[1, 6], c.table[2, :], c.table[3, 0], c.table[4, :4] = -1, c.n, 2 ** 31 - 1, -5, -(2 ** 31), -1
        q = _bounds(c, 4, rnd(g.standard_normal((c.rows, 4 * 128)), dt), kind)
        got = _attend(gpu, c, 4, dt, q)
        assert (got[c.rows:] == 3.0).all()
        k, v = c.values()
        want, mag, sens = (t[:c.rows] for t in lo.attention(q, 4, k, v, c.cu, c.lens, c.table, c.max_len))
        within(got[:c.rows], want, _bound(c, dt, want, mag, sens, np.abs(v).max()))
        assert (want == 0).all(axis=1).any()


def test_kv4_lengths_that_no_batch_should_have(gpu):
    """Lengths beyond the table, beyond the host's bound, negative ones and new rows beyond a length: held to what is there."""
    import torch
    g = np.random.default_rng(89)
    dt = "bf16"
    for lens in ([1000, 25, -7, 40], [2 ** 31 - 1, 0, -(2 ** 31), 48], [2 ** 31 - 5, 1, 2 ** 30, 47]):
        c = Pool(g, gpu, [40, 40, 40, 40], [2, 40, 3, 2], 1, 64, 16, dt)
        c.table = c.table[:, :3].copy()                       # 48 tokens a sequence at most
        c.lens = lens
        c.max_len = 47
        q = rnd(g.standard_normal((c.rows, 128)), dt)
        c.l = np.array(lens, np.int64).astype(np.int32)
        _check_attention(gpu, c, 2, dt, q)
        x = rnd(g.standard_normal((c.rows, 64)), dt)
        b, cache = c.load()
        X, p = dev(x, gpu, dt), tlq.params(x_dtype=tlq.BF16)
        tlq.kv4_append(X, X, b, cache, p)
        c.append(x, x)
        assert c.held()
        ko, vo = torch.full_like(X, 3.0), torch.full_like(X, 3.0)
        tlq.kv4_read(b, cache, p, ko, vo)
        for got, (codes, steps, turned) in ((ko, (c.kc, c.ks, False)), (vo, (c.vc, c.vs, True))):
            assert np.array_equal(host(got), rnd(lo.kv4_read(codes, steps, c.cu, lens, c.table, c.rows, c.max_len, turned), dt))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,most,group,page,kind", [
    ([40, 30], [5, 3], 1, 1, 16, ""), ([700, 40], [5, 20], 3, 2, 16, ""), ([3000, 2], [9, 2], 1, 4, 64, ""),
    ([300, 260, 9], [150, 260, 9], 40, 1, 64, "parts"), ([1500, 30], [200, 7], 130, 2, 32, "parts"), ([90, 70], [70, 70], 17, 2, 128, ""),
    ([10, 33], [20, 33], 12, 1, 16, "")])                    # (the last with rows before its first token)
def test_kv4_more_new_tokens_than_the_hosts_bound(gpu, dt, lens, new, most, group, page, kind):
    """Tokens behind a sequence's first max_new: their rows stay as they were, the cache takes none of them."""
    import torch
    g = np.random.default_rng([90, sum(lens), most])
    c = Pool(g, gpu, lens, new, 2, 64, page, dt)
    heads = 2 * group
    q = rnd(g.standard_normal((c.rows, heads * 64)), dt)
    c.max_new = most
    if kind == "parts":
        q = _bounds(c, heads, q, kind)
    got = _attend(gpu, c, heads, dt, q)
    taken = np.concatenate([np.arange(n) < most for n in new])
    assert (got[~taken] == 3.0).all() and not (got[taken] == 3.0).all(axis=1).any()
    k, v = c.values()
    want, mag, sens = lo.attention(q, heads, k, v, c.cu, c.lens, c.table, c.max_len)
    within(got[taken], want[taken], _bound(c, dt, want, mag, sens, np.abs(v).max())[taken])
    x = rnd(g.standard_normal((c.rows, 2 * 64)), dt)
    b, cache = c.load()
    p = tlq.params(x_dtype=CODE[dt])
    X = dev(x, gpu, dt)
    tlq.kv4_append(X, X, b, cache, p)
    c.append(x, x, most)
    assert c.held()
    out = torch.full_like(X, 3.0)
    tlq.kv4_read(b, cache, p, out)
    back = lo.kv4_read(c.kc, c.ks, c.cu, lens, c.table, c.rows, c.max_len, False)
    assert (host(out)[~taken] == 3.0).all() and np.array_equal(host(out)[taken], rnd(back[taken], dt))


@pytest.mark.parametrize("lens,new", [([700, 90], [1, 1]), ([700, 90], [40, 90])])
def test_kv4_tables_that_are_part_of_a_wider_one(gpu, lens, new):
    """Rows of a table further apart than they are long, what lies between them naming pages of no sequence; and a shared prefix."""
    g = np.random.default_rng(91)
    dt = "bf16"
    c = Pool(g, gpu, lens, new, 2, 128, 16, dt)
    c.table[1, :2] = c.table[0, :2]                           # (pages that neither call writes where 700 - 40 and 90 - 1 are new)
    q = rnd(g.standard_normal((c.rows, 4 * 128)), dt)
    narrow = _attend(gpu, c, 4, dt, q)
    _check_attention(gpu, c, 4, dt, q)
    b, cache = c.load()
    wide = dev(np.concatenate([c.table, np.full((2, 5), c.n - 1, np.int32)], 1), gpu)
    b = tlq.kv_batch(b.parts[0], b.parts[1], wide[:, :c.table.shape[1]], c.max_new, c.max_len)
    Q, p = dev(q, gpu, dt), tlq.params(x_dtype=CODE[dt])
    assert np.array_equal(host(tlq.kv4_attention(Q, 4, b, cache, p, dev(q, gpu, dt))), narrow)
    if new[1] == 1:
        x = rnd(g.standard_normal((c.rows, 2 * 128)), dt)
        X = dev(x, gpu, dt)
        tlq.kv4_append(X, X, b, cache, p)
        c.append(x, x)
        assert c.held()


def test_kv4_attention_of_very_many_sequences(gpu):
    """More blocks than one row of a grid has here, nearly all of them of sequences without tokens."""
    import torch
    g = np.random.default_rng(92)
    lens, new = np.zeros(65535, np.int64), np.zeros(65535, np.int64)
    lens[[0, 40000, 65527, 65534]], new[[0, 40000, 65527, 65534]] = [70, 33, 20, 150], [70, 1, 20, 20]
    c = Pool(g, gpu, lens.tolist(), new.tolist(), 1, 64, 16, "f16")
    q = np.full((2300, 64), np.nan, np.float32)                # (18 tiles a sequence by the host's bound)
    q[:c.rows] = rnd(g.standard_normal((c.rows, 64)), "f16")
    c.max_new, c.max_len = 2300, 2300
    _check_attention(gpu, c, 1, "f16", q)
    x = np.where(np.isnan(q), np.float32(1), q)
    c.max_new = 100                                           # (128 x 15 / 2048 + 1 blocks a sequence)
    b, cache = c.load()
    X = dev(x, gpu, "f16")
    tlq.kv4_append(X, X, b, cache, tlq.params())
    c.append(x, x, 100)
    assert c.held()


def test_kv4_attention_of_more_splits_than_lanes(gpu):
    """Parts of 256 keys of one sequence, and of a short one beside it."""
    g = np.random.default_rng(93)
    c = Pool(g, gpu, [40000, 300], [1, 1], 1, 128, 128, "bf16")
    _check_attention(gpu, c, 4, "bf16", rnd(g.standard_normal((2, 4 * 128)), "bf16"))


@pytest.mark.parametrize("new,kind", [(1, ""), (20, ""), (20, "tiles"), (20, "parts")])
def test_kv4_attention_of_many_keys_far_below_one(gpu, new, kind):
    """One key 2^22 times as heavy as each of 40,000 others, whose weights are no normal halves: together one percent of the sum,
    in the numerator and in the denominator alike."""
    g = np.random.default_rng(94)
    c = Pool(g, gpu, [40000 + new], [new], 1, 64, 64, "f16")
    for page in (2, 300, 600):                               # the heavy key in front, in the middle, near the end
        c.kc[:] = 0
        c.kc[c.table[0, page], 0, 5, :] = 7
        step = np.float16(rnd(np.float32(22 * np.log(2) / (7 * 8)), "bf16"))
        c.ks[:] = step
        c.vc[:] = np.clip(np.abs(c.vc), 1, 7)
        c.vc[c.table[0, page], 0, :, 5] = 0                  # what is left is the others' alone
        c.vs[:] = np.float16(0.03125)
        got = _attend(gpu, c, 2, "f16", _bounds(c, 2, np.ones((new, 128), np.float32), kind))[:new]
        k, v = c.values()
        want, mag, _ = lo.attention(np.ones((new, 128)), 2, k, v, c.cu, c.lens, c.table, c.max_len)
        # weights of about 2^-15 and 2^7: halves to 2^-11 and, those of subnormal ones, to 2^-10 (bits left of 2^-15); the score to 2^-17 of
        # itself, sums in 32 bits, a half of a small output
        within(got, want, want * (23 * 64 * U + 2.0 ** -10 + 2.0 ** -11 * 2.01 + 40000 / 16 * U) + TINY["f16"])


def test_kv4_attention_of_queries_near_the_types_largest(gpu):
    """bf16 queries of 2^126 and more with a scale that gives ordinary scores; subnormal ones."""
    g = np.random.default_rng(95)
    c = Pool(g, gpu, [70, 300], [2, 30], 1, 128, 16, "bf16")
    q = rnd(g.standard_normal((c.rows, 256)), "bf16")
    big = rnd(np.float32(2.0 ** 126) * (q / np.abs(q).max(axis=1, keepdims=True) * 1.9), "bf16")
    assert np.isfinite(big).all()
    _check_attention(gpu, c, 2, "bf16", big, scale=2.0 ** -125)
    _check_attention(gpu, c, 2, "bf16", rnd(big.astype(np.float64) * 2.0 ** -255, "bf16"))


def _winners(c, heads, q, scale):
    """(out, ok): the mean of the values of each row's largest score, ties among equal keys; ok where every other score lies further
    below it than floats can take (products of dh terms in 32 bits, and 64 binary orders)."""
    k, v = c.values()
    out, ok = np.zeros((c.rows, heads * c.dh)), np.zeros((c.rows, heads), bool)
    scale = scale or c.dh ** -0.5
    for s, n in enumerate(c.lens):
        ids = c.table[s, :-(-n // c.page)]
        for h in range(heads):
            keys = k[ids, h * c.kv // heads].reshape(-1, c.dh)[:n]
            vals = v[ids, h * c.kv // heads].transpose(0, 2, 1).reshape(-1, c.dh)[:n]
            for r in range(c.cu[s], c.cu[s + 1]):
                m = n - (c.cu[s + 1] - r) + 1
                terms = scale * keys[:m] * q[r, h * c.dh:(h + 1) * c.dh].astype(np.float64)
                z, sens = terms.sum(1), np.abs(terms).sum(1).max()
                top = z == z.max()
                out[r, h * c.dh:(h + 1) * c.dh] = vals[:m][top].mean(0)
                ok[r, h] = top.all() or z.max() - z[~top].max() > 64 + 4 * (c.dh + 8) * U * sens
    return out, np.repeat(ok, c.dh, 1)


@pytest.mark.parametrize("kind", ["", "tiles", "parts"])
@pytest.mark.parametrize("dt,size,scale,dh", [
    ("f16", 6e4, 0.0, 128), ("f16", 6e4, -3e4, 128), ("bf16", 2.0 ** 28, 0.0, 128), ("bf16", 2.0 ** 60, 0.0, 128), ("bf16", 2.0 ** 101, 0.0, 128),
    ("bf16", 2.0 ** 126, 0.0, 128), ("bf16", 2.0 ** 126, -2.0 ** 60, 128), ("f16", 6e4, 0.0, 64), ("bf16", 2.0 ** 101, 0.0, 64)])
def test_kv4_attention_of_scores_of_any_size(gpu, kind, dt, size, scale, dh):
    """Scores (2^28 to 2^192) whose neighbours as floats lie many binary orders on, or that no float is, of both signs or all below
    zero: the largest takes all of the weight, keys that are equal share it.  Rows with ordinary scores beside them keep their bits."""
    g = np.random.default_rng(101)
    c = Pool(g, gpu, [700, 300, 3], [5, 40, 3], 2, dh, 16, dt)
    for s, n in enumerate(c.lens):                             # the second half of a sequence has the keys of the first again
        for t in range(n // 2):
            a, b = (c.table[s, t // 16], slice(None), t % 16), (c.table[s, (t + n // 2) // 16], slice(None), (t + n // 2) % 16)
            c.kc[b], c.ks[b] = c.kc[a], c.ks[a]
    c.kc[:, 0] = -np.abs(c.kc[:, 0])
    if dt == "f16":
        c.ks[:] = np.minimum(c.ks.astype(np.float32) * 2.0 ** 14, 8160.0).astype(np.float16)      # (eight times 8192 is no half)
    q = g.standard_normal((c.rows, 4 * dh))
    q[::4, :2 * dh] = np.abs(q[::4, :2 * dh]) + 0.1                  # (with the keys of head 0: no score above zero)
    plain = rnd(q * (1e-4 if dt == "f16" else 1.0), dt)
    loud = rnd(q / np.abs(q).max(axis=1, keepdims=True) * size, dt)
    loud[1::2] = plain[1::2]
    far = np.arange(c.rows) % 2 == 0
    want, ok = _winners(c, 4, loud, scale)
    assert ok[far].mean() > 0.9
    got = _attend(gpu, c, 4, dt, _bounds(c, 4, loud, kind), scale)[:c.rows]
    assert np.isfinite(got[far]).all()
    # (of one weight, or a few that are equal: sums and quotient in 32 bits, the output)
    within(got[ok & far[:, None]], want[ok & far[:, None]], (np.abs(want) * (HALF[dt] * 1.001 + 8 * U) + TINY[dt] * 1.01)[ok & far[:, None]])
    if scale == 0.0:
        quiet = _attend(gpu, c, 4, dt, _bounds(c, 4, plain, kind), scale)[:c.rows]
        assert np.isfinite(quiet).all() and np.array_equal(got[~far], quiet[~far])


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new,kind", [(1, ""), (20, ""), (20, "tiles"), (20, "parts"), (150, ""), (150, "tiles"), (150, "parts")])
def test_kv4_attention_of_queries_that_are_not_finite(gpu, dt, new, kind):
    """An infinity or a NaN anywhere in a query makes its head NaN, whichever sign the keys have there, and no other head; a row
    that sees no key gives zeros still.  Split and unsplit."""
    g = np.random.default_rng(96)
    for length in (200, 3000):
        c = Pool(g, gpu, [length, 40], [new, 1], 2, 64, 32, dt)
        c.kc[:, 0] = np.abs(c.kc[:, 0]) % 8
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


def test_kv4_pools_beyond_two_to_the_31(gpu):
    """Pages whose words lie further than 2^31 and 2^32 bytes into the pool."""
    import torch
    kv, dh, page, n = 4, 128, 256, (1 << 16) + 300            # 65,536 bytes a page: 4.3 GB of keys, as many of values
    kc, vc = (torch.empty((n, kv) + sh, dtype=torch.int32, device=gpu) for sh in ((page, dh // 8), (dh, page // 8)))
    ks, vs = (torch.empty((n, kv) + sh, dtype=torch.float16, device=gpu) for sh in ((page, 4), (4, page)))
    cache = tlq.kv4_cache(kc, ks, vc, vs)
    near = tlq.kv4_cache(*[t[:8].clone() for t in (kc, ks, vc, vs)])
    far = np.array([[n - 1, 40000, 5], [65537, 32769, 3]], np.int32)
    cu, lens = np.array([0, 600, 1100], np.int32), np.array([600, 500], np.int32)
    X = torch.randn((1100, kv * dh), device=gpu).half()
    p = tlq.params()
    outs = []
    for table, pool in ((far, cache), (np.array([[0, 1, 2], [3, 4, 5]], np.int32), near)):
        t = dev(table, gpu)
        batch = tlq.kv_batch(dev(cu, gpu), dev(lens, gpu), t, 600, 600)
        tlq.kv4_append(X, X, batch, pool, p)
        Q = X.repeat(1, 2).contiguous()
        outs.append(tlq.kv4_attention(Q, 8, batch, pool, p, torch.empty_like(Q)))
        k, v = torch.empty_like(X), torch.empty_like(X)
        tlq.kv4_read(batch, pool, p, k, v)
        one = tlq.kv_batch(dev(np.array([0, 1, 2], np.int32), gpu), dev(lens, gpu), t, 1, 600)
        tlq.kv4_append(X[:2], X[2:4], one, pool, p)
        outs += [tlq.kv4_attention(Q[:2], 8, one, pool, p, torch.empty_like(Q[:2])), k, v]
    for a, b in zip(outs[:4], outs[4:]):
        assert torch.equal(a, b) and bool(a.isfinite().all())
    assert torch.equal(outs[2], outs[3])


# ------------------------------------------------------------------ together
def _weights(gpu, g, co, ci, dt):
    import torch
    W = dev(rnd(g.standard_normal((co, ci)) * ci ** -0.5, dt), gpu, dt)
    codes, steps = torch.empty((co, -(-ci // 128) * 128), dtype=torch.int8, device=gpu), torch.empty(co, device=gpu)
    tlq.row_codes(W, 8, tlq.params(x_dtype=CODE[dt]), codes, steps)
    return codes, steps


class Block:
    """A vision-language decoder block in low bits, as a program runs it; `see` is called with every operator's name, inputs and
    outputs."""

    def __init__(self, gpu, g, d, heads, kv, dh, ffn, dt):
        self.d, self.heads, self.kv, self.dh, self.ffn, self.dt, self.gpu = d, heads, kv, dh, ffn, dt, gpu
        self.p = tlq.params(bits=8, group=0, symmetric=1, act_bits=8, x_dtype=CODE[dt], yref_dtype=CODE[dt])
        self.qkv, self.o = _weights(gpu, g, (heads + 2 * kv) * dh, d, dt), _weights(gpu, g, d, heads * dh, dt)
        self.gate, self.up, self.down = _weights(gpu, g, ffn, d, dt), _weights(gpu, g, ffn, d, dt), _weights(gpu, g, d, ffn, dt)
        self.bias = dev(0.3 * g.standard_normal((heads + 2 * kv) * dh).astype(np.float32), gpu)
        self.n1, self.n2 = (dev(np.exp(0.2 * g.standard_normal(d)).astype(np.float32), gpu) for _ in range(2))
        self.inv = dev(1e4 ** (-np.arange(dh // 2) / (dh // 2)), gpu)
        self.axis = dev((np.arange(dh // 2) % 3).astype(np.int32), gpu)

    def new(self, n, m):
        import torch
        return torch.empty((n, m), dtype=tt(self.dt), device=self.gpu)

    def codes(self, n, c):
        import torch
        return torch.empty((n, -(-c // 128) * 128), dtype=torch.int8, device=self.gpu), torch.empty(n, device=self.gpu)

    def run(self, h, z, pos, batch, cache, work, see=lambda *a: None):
        """h + z, the block, and the stream behind it with the last product added."""
        n, d, dh, nq, nk = h.shape[0], self.d, self.dh, self.heads * self.dh, self.kv * self.dh
        c, s = self.codes(n, d)
        h0 = self.new(n, d)
        tlq.add_norm_codes(h, self.n1, self.p, c, s, Z=z, H_out=h0)
        see("norm", (h, z, self.n1), (h0, c, s))
        qkv = tlq.linear_codes(c, s, d, *self.qkv, self.p, self.new(n, nq + 2 * nk), bias=self.bias, workspace=work)
        see("linear", (c, s, d, self.qkv, self.bias, 0, None, False), qkv)
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
        before = q.clone()
        tlq.qk_norm_rope_axes(q, k, dh, pos, self.axis, self.inv, self.p, q, k, norm=False)
        see("rope", (before, pos), q)
        tlq.kv4_append(k, v, batch, cache, self.p)
        see("append", (k, v), None)
        a = tlq.kv4_attention(q, self.heads, batch, cache, self.p, self.new(n, nq), workspace=work)
        see("attention", q, a)
        c, s = self.codes(n, nq)
        tlq.row_codes(a, 8, self.p, c, s)
        residual = h0.clone()
        tlq.linear_codes(c, s, nq, *self.o, self.p, h0, R=h0, workspace=work)            # onto the stream
        see("linear", (c, s, nq, self.o, None, 0, residual, False), h0)
        c, s = self.codes(n, d)
        tlq.add_norm_codes(h0, self.n2, self.p, c, s)
        see("norm", (h0, None, self.n2), (h0, c, s))
        up = tlq.linear_codes(c, s, d, *self.up, self.p, self.new(n, self.ffn), workspace=work)
        was = up.clone()
        tlq.linear_codes(c, s, d, *self.gate, self.p, up, act=tlq.ACT_SILU, R=up, mul=True, workspace=work)
        see("linear", (c, s, d, self.gate, None, 1, was, True), up)
        c, s = self.codes(n, self.ffn)
        tlq.row_codes(up, 8, self.p, c, s)
        y = tlq.linear_codes(c, s, self.ffn, *self.down, self.p, self.new(n, d), R=h0, workspace=work)
        see("linear", (c, s, self.ffn, self.down, None, 0, h0, False), y)
        return y


@pytest.mark.parametrize("dt,heads,kv,dh", [("bf16", 4, 2, 128), ("f16", 6, 1, 64)])
def test_a_block_in_low_bits(gpu, dt, heads, kv, dh):
    """Prompts of three sequences, images among them, and four steps of single tokens through a whole block; every operator is held
    to the oracle on the inputs that it met."""
    import torch
    g = np.random.default_rng([97, heads])
    d, ffn, page = 256, 384, 16
    block = Block(gpu, g, d, heads, kv, dh, ffn, dt)
    prompt = [19, 33, 7]
    c = Pool(g, gpu, [n + 4 for n in prompt], prompt, kv, dh, page, dt)
    c.load()
    cache, table = tlq.kv4_cache(*c.t), dev(c.table, gpu)
    lens = np.zeros(3, np.int32)
    work = torch.empty(1 << 24, dtype=torch.uint8, device=gpu)
    seen = set()
    for counts in [prompt] + [[1, 1, 1]] * 4:
        n = sum(counts)
        lens = lens + np.array(counts, np.int32)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        at = np.concatenate([np.arange(l - m, l) for l, m in zip(lens, counts)])
        pos = np.stack([at, at // 4, at % 4]).astype(np.int32) if n > 3 else np.stack([at] * 3).astype(np.int32)
        batch = tlq.kv_batch(dev(cu, gpu), dev(lens.astype(np.int32), gpu), table, max(counts), 64)

        def see(name, a, out):
            seen.add(name)
            if name == "norm":
                h, z, w = a
                want = lo.add_norm_codes(host(h).astype(np.float32), None if z is None else host(z).astype(np.float32), w.cpu().numpy(), 1e-6, 8, dt == "bf16")
                assert np.array_equal(host(out[0]), want[0]) and np.array_equal(out[1].cpu().numpy()[:, :h.shape[1]], want[1]) and np.array_equal(out[2].cpu().numpy(), want[2])
            elif name == "linear":
                codes, steps, ci, (wc, ws), bias, kind, r, mul = a
                r = None if r is None else host(r)
                want, prod, v, act = lo.linear_codes(codes.cpu().numpy()[:, :ci], steps.cpu().numpy(), wc.cpu().numpy()[:, :ci], ws.cpu().numpy(),
                                                     None if bias is None else bias.cpu().numpy(), kind, r, mul)
                within(host(out), want, _linear_bound(prod, v, act, want, kind, r, mul, dt))
            elif name == "rope":
                want = lo.norm_rope_axes(host(a[0]), dh, a[1].cpu().numpy(), np.arange(dh // 2) % 3, block.inv.cpu().numpy(), norm=False)
                within(host(out), want, np.abs(want) * HALF[dt] * 1.001 + 2e-5 * np.abs(want).max())
            elif name == "append":
                c.cu, c.lens, c.max_len = cu, lens, 64
                c.append(host(a[0]).astype(np.float32), host(a[1]).astype(np.float32))
                assert c.held()
            else:
                k, v = c.values()
                want, mag, sens = lo.attention(host(a), heads, k, v, cu, lens, c.table, 64)
                within(host(out), want, _bound(c, dt, want, mag, sens, np.abs(v).max()))
        h, z = (dev(rnd(g.standard_normal((n, d)), dt), gpu, dt) for _ in range(2))
        y = block.run(h, z, dev(pos, gpu), batch, cache, work, see)
        assert bool(torch.isfinite(y).all())
    assert seen == {"norm", "linear", "rope", "append", "attention"}


def test_a_step_as_a_graph(gpu):
    """One step of single tokens through the block, captured; lengths and inputs change between replays, eager work lies between them,
    and a second graph shares the workspace."""
    import torch
    g = np.random.default_rng(98)
    heads, kv, dh, page, dt = 8, 2, 128, 64, "bf16"
    d = heads * dh
    block = Block(gpu, g, d, heads, kv, dh, 512, dt)
    c = Pool(g, gpu, [900, 700], [1, 1], kv, dh, page, dt)
    c.load()
    cache = tlq.kv4_cache(*c.t)
    cu, lens, table = dev(c.cu, gpu), dev(np.array([700, 500], np.int32), gpu), dev(c.table, gpu)
    pos = torch.zeros((3, 2), dtype=torch.int32, device=gpu)
    batch = tlq.kv_batch(cu, lens, table, 1, 900)
    h, z = (torch.empty((2, d), dtype=tt(dt), device=gpu) for _ in range(2))
    work = torch.empty(1 << 24, dtype=torch.uint8, device=gpu)
    k, v = (torch.empty((2, kv * dh), dtype=tt(dt), device=gpu) for _ in range(2))

    def step():
        y = block.run(h, z, pos, batch, cache, work)
        tlq.kv4_read(batch, cache, block.p, k, v)
        return y

    def fresh():
        for t in (h, z):
            t.copy_(dev(rnd(g.standard_normal((2, d)), dt), gpu, dt))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fresh()
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(step())
    saved = [t.clone() for t in c.t]
    for i in range(4):
        fresh()
        lens.copy_(dev(np.array([701 + 60 * i, 501 + i], np.int32), gpu))
        pos.copy_((lens - 1).expand(3, 2))
        for t, o in zip(c.t, saved):
            t.copy_(o)
        y = step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, k, v, *c.t)]
        for graph, out in zip(graphs, outs):
            for t, o in zip(c.t, saved):
                t.copy_(o)
            work.fill_(0xFF)
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for got, e in zip((out, k, v, *c.t), want):
                assert torch.equal(got, e)


def test_two_streams_at_once(gpu):
    """Calls on two streams with workspaces and outputs of their own do not meet, and run in their stream's order."""
    import torch
    g = np.random.default_rng(99)
    p = tlq.params()
    c = Pool(g, gpu, [3000, 100], [1, 1], 2, 128, 64, "f16")
    b, cache = c.load()
    codes, steps, w, ws = _linear_case(g, 40, 2056, 9001)
    X, S, W, WS = _padded(codes, gpu), dev(steps, gpu), _padded(w, gpu), dev(ws, gpu)
    q = dev(rnd(g.standard_normal((2, 8 * 128)), "f16"), gpu, "f16")
    H = dev(rnd(g.standard_normal((300, 4104)), "f16"), gpu, "f16")

    def once():
        y = tlq.linear_codes(X, S, 2056, W, WS, p, torch.empty((40, 9008), dtype=torch.float16, device=gpu)[:, :9001], act=tlq.ACT_GELU_ERF)
        a = tlq.kv4_attention(q, 8, b, cache, p, torch.empty_like(q))
        out, cd, st = torch.empty_like(H), torch.empty((300, 4224), dtype=torch.int8, device=gpu), torch.empty(300, device=gpu)
        tlq.add_norm_codes(H, None, p, cd, st, Z=H, H_out=out)
        k, v = (torch.empty((2, 256), dtype=torch.float16, device=gpu) for _ in range(2))
        tlq.kv4_read(b, cache, p, k, v)
        return y, a, out, cd, st, k, v
    want = [t.clone() for t in once()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(once())
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(x, y) for x, y in zip(o, want))


def test_single_rows_of_any_stride(gpu):
    """The stride of a matrix of one row is never used; one token's positions may be a column of a wider matrix."""
    import torch
    g = np.random.default_rng(100)
    p = tlq.params()
    h = dev(rnd(g.standard_normal((1, 256)), "f16"), gpu, "f16")
    column = h.reshape(256, 1).t()                            # [1, 256] with strides of one
    outs = []
    for t in (h, column):
        codes, steps = torch.empty((1, 256), dtype=torch.int8, device=gpu), torch.empty(1, device=gpu)
        tlq.add_norm_codes(t, None, p, codes, steps)
        outs += [codes, steps]
    assert column.stride() == (1, 1) and torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    pos = torch.arange(30, dtype=torch.int32, device=gpu).reshape(3, 10)
    axis, inv = torch.arange(32, device=gpu).to(torch.int32) % 3, dev(1e3 ** (-np.arange(32) / 32), gpu)
    a, b = (tlq.qk_norm_rope_axes(h[:, :128], h[:, 128:], 64, t, axis, inv, p, torch.empty_like(h[:, :128]), torch.empty_like(h[:, 128:]))
            for t in (pos[:, 4:5], pos[:, 4:5].contiguous()))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
