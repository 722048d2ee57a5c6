"""Linear maps with an epilogue, norms around a gated residual sum, log
probabilities of labels and their gradients against plain 64-bit
implementations (needs an MI355X).

Tolerances follow from the arithmetic: u = 2^-24 is half a step of fp32, a sum
of n terms in any order is off by at most n u times the sum of their sizes
(matrix cores: twice that, their adder may truncate), and the stored result
by half a step of its type.  Errors of inputs go through each formula to first
order.
"""
import math

import pytest
import torch

import paper_2607_17374_amd as T
from paper_2607_17374_amd import _native as N
from tests.test_gpu_rowops import BF16, DTYPES, F16, F32, HALF, TINY, U, close, normal, note, ranges, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cuda(t):
    return None if t is None else t.cuda()


# ------------------------------------------------------------------ linear --

ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def phi_cdf(z):
    return 0.5 * torch.erfc(-z / math.sqrt(2.0))


def tanh_parts(z):
    """u with gelu_tanh(z) = z sigmoid(u), and its slope."""
    a = 2.0 * math.sqrt(2.0 / math.pi)
    return a * (z + 0.044715 * z ** 3), a * (1.0 + 3 * 0.044715 * z * z)


def sigmoid_error(u):
    """The sigmoid to 8 u, its argument to 4 u of its size."""
    q = torch.sigmoid(u)
    return q, q * (8 * U + 4 * U * u.abs() * (1 - q)) + 2.0 ** -126


def act_of(z, tz, act):
    """Activation of z known to tz, and how far the fp32 value may be off.  No
    slope passes 1.13."""
    if act == "relu":
        return z.clamp(min=0), tz
    if act == "silu":
        y = z * torch.sigmoid(z)
        return y, 1.13 * tz + 16 * U * y.abs()
    if act == "gelu":
        # the tail Phi(-|z|) to 10 u and 3 u z^2 of itself, 1 minus it to u
        tail = phi_cdf(-z.abs())
        y = z * phi_cdf(z)
        return y, 1.13 * tz + z.abs() * (tail * (10 + 3 * z * z) * U + (z > 0) * U) + 2 * U * y.abs()
    if act == "gelu_tanh":
        u, _ = tanh_parts(z)
        q, eq = sigmoid_error(u)
        y = z * q
        return y, 1.13 * tz + z.abs() * eq + 2 * U * y.abs()
    return z, tz


def slope_of(z, act):
    """act'(z) and how far the fp32 value may be off."""
    if act == "relu":
        return (z > 0).double(), torch.zeros_like(z)
    if act == "silu":
        q, eq = sigmoid_error(z)
        s = q * (1 + z * (1 - q))
        return s, eq * (1 + z.abs()) + 6 * U * (q + z.abs() * q * (1 - q))
    if act == "gelu":
        tail, density = phi_cdf(-z.abs()), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        s = phi_cdf(z) + z * density
        e = tail * (10 + 3 * z * z) * U + (z > 0) * U + z.abs() * density * (6 + 3 * z * z) * U
        return s, e + 2 * U * (phi_cdf(z) + z.abs() * density)
    if act == "gelu_tanh":
        u, du = tanh_parts(z)
        q, eq = sigmoid_error(u)
        s = q * (1 + z * (1 - q) * du)
        return s, eq * (1 + z.abs() * du) + 8 * U * (q + z.abs() * q * (1 - q) * du)
    return torch.ones_like(z), torch.zeros_like(z)


def linear_reference(x, w, b, res, act):
    """(z, its tolerance, out, its tolerance) in 64 bits."""
    k = x.shape[1]
    z = x.double() @ w.double()
    tz = 2 * (k + 2) * U * (x.double().abs() @ w.double().abs())
    if b is not None:
        z = z + b.double()
        tz = tz + 2 * U * (z.abs() + b.double().abs())
    y, ty = act_of(z, tz, act)
    if res is not None:
        y = y + res.double()
        ty = ty + 2 * U * (y.abs() + res.double().abs())
    return z, tz, y, ty


LINEAR = [  # rows, d_in, d_out
    (1, 1, 1), (3, 5, 7), (2, 9, 1), (1, 1024, 1024), (3, 64, 64), (17, 130, 47), (128, 64, 128), (129, 200, 65),
    (200, 1000, 136), (513, 256, 256), (1000, 72, 300), (64, 4096, 96), (16, 2050, 40), (5, 8, 2000), (700, 33, 90),
    (300, 520, 264), (0, 16, 8), (1, 2048, 8200), (16, 31, 4100), (17, 96, 8193), (32, 300, 33), (33, 513, 70), (64, 40, 9000),
    (5, 7, 3), (48, 1000, 7), (65, 1000, 7), (9, 4, 4), (3, 4100, 70), (20, 3000, 24), (32, 9000, 10),
    (1, 2049, 1),
]


def check_linear(x, w, b, res, act, out_dtype, pre, **where):
    r = T.linear(cuda(x), cuda(w), cuda(b), cuda(res), act=act, out_dtype=out_dtype, pre=pre, **where)
    z, tz, y, ty = linear_reference(x, w, b, res, act)
    out, got_z = r if pre else (r, None)
    assert out.dtype == out_dtype
    close(out, y, ty, out_dtype, "out")
    if pre:
        assert got_z.dtype == x.dtype
        close(got_z, z, tz, x.dtype, "pre")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LINEAR)))
def test_linear(dtype, case):
    m, k, n = LINEAR[case]
    for i in range(2):
        act, out_dtype = ACTS[(case + 2 * i) % 5], [dtype, F32][(case + i) % 2]
        note(f"linear {dtype} m={m} k={k} n={n} {act} -> {out_dtype}")
        x, w = normal((m, k), dtype, case), normal((k, n), dtype, case + 1, k ** -0.5)
        b = normal((n,), F32, case + 2) if (case + i) % 3 else None
        res = normal((m, n), out_dtype, case + 3) if (case + i) % 2 else None
        check_linear(x, w, b, res, act, out_dtype, (case + i) % 3 != 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,n,pad,lead", [(64, 64, 64, 8, 8), (70, 64, 64, 3, 1), (300, 40, 72, 0, 1),
                                            (33, 17, 9, 2, 0), (150, 128, 260, 4, 4), (9, 600, 66, 1, 2),
                                            (520, 264, 520, 8, 0), (520, 264, 520, 5, 3)])
def test_linear_strided(dtype, m, k, n, pad, lead):
    note(f"linear strided {dtype} m={m} k={k} n={n} pad={pad} lead={lead}")
    x, w, b = normal((m, k), dtype, 1), normal((k, n), dtype, 2, k ** -0.5), normal((n,), F32, 3)
    res = normal((m, n), dtype, 4)
    wide = torch.full((m, lead + n + pad), 7.0, dtype=dtype, device="cuda")
    out = wide[:, lead:lead + n]
    got, pre = T.linear(strided(x, pad, lead), w.cuda(), b.cuda(), strided(res, pad, lead), act="silu", out=out, pre=True)
    assert got is out
    z, tz, y, ty = linear_reference(x, w, b, res, "silu")
    close(out, y, ty, dtype, "out")
    close(pre, z, tz, dtype, "pre")
    assert (torch.cat([wide[:, :lead], wide[:, lead + n:]], 1) == 7.0).all()
    grad = normal((m, n), dtype, 5)
    check_linear_grad(x, w, grad, "silu", F32, pre, strided(x, pad, lead), strided(grad, pad, lead),
                      strided(pre.cpu(), pad, lead))


def check_linear_grad(x, w, grad, act, weight_dtype, pre, xs=None, gs=None, zs=None):
    """Against the formula at the pre that the call is given."""
    m, n = grad.shape
    xs, gs = cuda(x) if xs is None else xs, cuda(grad) if gs is None else gs
    zs = (None if pre is None else pre.cuda()) if zs is None else zs
    dx, dw, db = T.linear_grad(gs, xs, w.cuda(), zs, act=act, weight_dtype=weight_dtype)
    slope, ts = slope_of(torch.zeros(m, n).double() if pre is None else pre.double().cpu(), act)
    g = grad.double()
    dz = g * slope
    t32 = g.abs() * ts + (0 if act in ("none", "relu") else U) * dz.abs()
    # rounded to the operands' type, but where it is grad itself
    t = t32 if act in ("none", "relu") else t32 + HALF[x.dtype] * (dz.abs() + t32) + TINY[x.dtype]
    size = dz.abs() + t
    W, X = w.double(), x.double()
    close(dx, dz @ W.t(), t @ W.abs().t() + 2 * (n + 2) * U * (size @ W.abs().t()), x.dtype, "dx")
    close(dw, X.t() @ dz, X.abs().t() @ t + 2 * (m + 2) * U * (X.abs().t() @ size), weight_dtype, "dweight")
    close(db, dz.sum(0), t32.sum(0) + m * U * (dz.abs() + t32).sum(0), F32, "dbias")
    for only in ("x", "weight", "bias"):
        r = T.linear_grad(gs, xs, w.cuda(), zs, act=act, need=(only,), weight_dtype=weight_dtype)
        for one, every, name in zip(r, (dx, dw, db), ("x", "weight", "bias")):
            assert (one is None) == (name != only)
            assert one is None or torch.equal(one, every)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LINEAR)))
def test_linear_grad(dtype, case):
    m, k, n = LINEAR[case]
    for i in range(2):
        act, weight_dtype = ACTS[(case + 2 * i) % 5], [F32, dtype][(case + i) % 2]
        note(f"linear_grad {dtype} m={m} k={k} n={n} {act} -> {weight_dtype}")
        x, w, grad = normal((m, k), dtype, case), normal((k, n), dtype, case + 1, k ** -0.5), normal((m, n), dtype, case + 2)
        pre = None if act == "none" else normal((m, n), dtype, case + 3, 2.0)
        check_linear_grad(x, w, grad, act, weight_dtype, pre)


LARGE = [  # rows, d_in, d_out: several tiles every way, rests of tiles and stages
    (1024, 512, 1024), (1100, 1000, 520), (2049, 264, 1032), (770, 2056, 776), (515, 1032, 2056), (4100, 136, 264),
    (40_003, 64, 72), (9000, 256, 512),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LARGE)))
def test_linear_large(dtype, case):
    m, k, n = LARGE[case]
    act, out_dtype = ACTS[case % 5], [dtype, F32][case % 2]
    note(f"linear large {dtype} m={m} k={k} n={n} {act} -> {out_dtype}")
    x, w, b = normal((m, k), dtype, case), normal((k, n), dtype, case + 1, k ** -0.5), normal((n,), F32, case + 2)
    res = normal((m, n), out_dtype, case + 3) if case % 3 else None
    check_linear(x, w, b, res, act, out_dtype, case % 2 == 0)
    pre = None if act == "none" else normal((m, n), dtype, case + 4, 2.0)
    check_linear_grad(x, w, normal((m, n), dtype, case + 5), act, [F32, dtype][case % 2], pre)


WIDE = [  # rows, d_in, d_out of products in tiles of 256 x 256 (fp32: 128 x 128): a single partial
    # round of tiles, whole rounds and a rest, a rest too large to cut, rests of
    # every tile and stage
    (2049, 1032, 2904), (5000, 520, 3208), (16_500, 264, 1480), (772, 4100, 2060), (30_001, 256, 840),
]


@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("m,k,n", [(260, 8196, 1000), (30_000, 260, 264), (999, 2052, 1004), (2048, 1024, 1024)])
def test_linear_wide_f32(m, k, n, out_dtype):
    """The smallest that go through these tiles."""
    note(f"linear wide float32 m={m} k={k} n={n} -> {out_dtype}")
    x, w, b = normal((m, k), F32, m), normal((k, n), F32, m + 1, k ** -0.5), normal((n,), F32, m + 2)
    check_linear(x, w, b, normal((m, n), out_dtype, m + 3), "silu", out_dtype, True)
    if out_dtype == F32:
        check_linear_grad(x, w, normal((m, n), F32, m + 4), "silu", F32, normal((m, n), F32, m + 5, 2.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(WIDE)))
def test_linear_wide(dtype, case):
    m, k, n = WIDE[case]
    act, out_dtype = ACTS[case % 5], [dtype, F32][case % 2]
    note(f"linear wide {dtype} m={m} k={k} n={n} {act} -> {out_dtype}")
    x, w, b = normal((m, k), dtype, case), normal((k, n), dtype, case + 1, k ** -0.5), normal((n,), F32, case + 2)
    res = normal((m, n), out_dtype, case + 3) if case % 3 != 1 else None
    check_linear(x, w, b, res, act, out_dtype, case % 2 == 0)
    pre = None if act == "none" else normal((m, n), dtype, case + 4, 2.0)
    check_linear_grad(x, w, normal((m, n), dtype, case + 5), act, [F32, dtype][case % 2], pre)


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_wide_strided(dtype):
    """Rows that are wide apart, whose surroundings are NaN, and special values
    in the last rows and columns."""
    note(f"linear wide strided {dtype}")
    m, k, n = 2050, 1040, 2912
    x, w, b = normal((m, k), dtype, 1), normal((k, n), dtype, 2, k ** -0.5), normal((n,), F32, 3)
    wide = torch.full((m, n + 24), 7.0, dtype=dtype, device="cuda")
    out = wide[:, 8:8 + n]
    got, pre = T.linear(strided(x, 8, 16), w.cuda(), b.cuda(), strided(b.to(dtype).expand(m, n), 16, 8), act="relu", out=out, pre=True)
    z, tz, y, ty = linear_reference(x, w, b, b.to(dtype).expand(m, n), "relu")
    close(out, y, ty, dtype, "out")
    close(pre, z, tz, dtype, "pre")
    assert (torch.cat([wide[:, :8], wide[:, 8 + n:]], 1) == 7.0).all()
    x[:], w[:] = 1, 1
    x[1, 0], x[m - 1, k - 1], w[3, n - 1] = math.inf, math.nan, -math.inf
    out = T.linear(strided(x, 8, 0), w.cuda(), out_dtype=F32).cpu()
    rest = torch.ones(m, dtype=torch.bool)
    rest[1] = rest[m - 1] = False
    assert (out[rest][:, :n - 1] == k).all() and (out[rest][:, n - 1] == -math.inf).all()
    assert (out[1, :n - 1] == math.inf).all() and torch.isnan(out[1, n - 1]) and torch.isnan(out[m - 1]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
def test_linear_wide_at_odd_addresses(dtype, out_dtype):
    """What the large products write and the residual they read lie at any
    address of a value, an odd number of values apart; only x and the weight
    choose them."""
    note(f"linear wide at odd addresses {dtype} -> {out_dtype}")
    m, k, n = 1050, 1040, 5808
    x, w, b = normal((m, k), dtype, 1), normal((k, n), dtype, 2, k ** -0.5), normal((n,), F32, 3)
    res = normal((m, n), out_dtype, 4)
    wide, wide_z = (torch.full((m, n + 4), 7.0, dtype=t, device="cuda") for t in (out_dtype, dtype))
    out, z, rs = wide[:, 1:1 + n], wide_z[:, 3:3 + n], strided(res, 2, 3)
    xd, wd, bd = x.cuda(), w.cuda(), b.cuda()
    code = {F32: N.F32, BF16: N.BF16, F16: N.F16}
    nbytes = N.lib().taurus_linear_bytes(code[dtype], m, k, n)
    work = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    N.check(N.lib().taurus_linear(xd.data_ptr(), code[dtype], m, k, k, wd.data_ptr(), n, bd.data_ptr(), rs.data_ptr(),
                                  rs.stride(0), N.ACT_GELU, out.data_ptr(), code[out_dtype], out.stride(0), z.data_ptr(),
                                  z.stride(0), work.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream), "taurus_linear")
    want_z, tz, y, ty = linear_reference(x, w, b, res, "gelu")
    close(out, y, ty, out_dtype, "out")
    close(z, want_z, tz, dtype, "pre")
    for t, at in ((wide, 1), (wide_z, 3)):
        assert (torch.cat([t[:, :at], t[:, at + n:]], 1) == 7.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(6))
def test_linear_few_rows_into_many_columns(dtype, case):
    """17 to 32 rows (and 16, one block) with the most columns a lane and sixteen
    waves: from 512 values on into at least 8,192 columns, fp32 4,096."""
    m, k, n = [(32, 1024, 8192), (17, 512, 8200), (25, 4100, 8195), (32, 2048, 16_400), (16, 777, 8300), (31, 515, 4099)][case]
    act, out_dtype = ACTS[case % 5], [dtype, F32][case % 2]
    note(f"linear few rows {dtype} m={m} k={k} n={n} {act} -> {out_dtype}")
    x, w, b = normal((m, k), dtype, case), normal((k, n), dtype, case + 1, k ** -0.5), normal((n,), F32, case + 2)
    check_linear(x, w, b, normal((m, n), out_dtype, case + 3) if case % 3 else None, act, out_dtype, case % 2 == 0)
    pre = None if act == "none" else normal((m, n), dtype, case + 4, 2.0)
    check_linear_grad(x, w, normal((m, n), dtype, case + 5), act, F32, pre)


def whole(shape, dtype, seed):
    """Whole numbers from -2 to 2, none of them zero."""
    g = torch.Generator().manual_seed(seed)
    return torch.tensor([-2.0, -1.0, 1.0, 2.0])[torch.randint(0, 4, shape, generator=g)].to(dtype)


EXACT = [  # rows, d_in, d_out: contractions cut into many parts and joined, long slope passes, rests of rows, stages and
    # tiles, few rows with a long contraction, the widest outputs of few rows
    (30_001, 256, 840), (40_003, 64, 72), (16_500, 264, 1480), (300_007, 3, 5), (70_001, 33, 47), (100_001, 16, 8),
    (9_999, 520, 264), (20_480, 256, 256), (4_097, 1032, 1000), (257, 8200, 300), (2_000, 96, 1),
    (40, 9000, 50), (20, 9000, 40), (32, 4096, 8200), (17, 513, 16_387), (31, 512, 4096), (3, 20_000, 70), (16, 6000, 9),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(EXACT)))
def test_linear_exact(dtype, case):
    """Sums of whole numbers, which fp32 holds exactly (up to 4 a term, below
    2^24) in whatever order and parts they are added: a row, column or term that
    is lost, doubled or of a neighbour shows in an output that is not equal."""
    m, k, n = EXACT[case]
    act = ["none", "relu"][case % 2]
    note(f"linear exact {dtype} m={m} k={k} n={n} {act}")
    assert 4 * max(m, k, n) + 4 < 2 ** 24
    x, w, grad = whole((m, k), dtype, case), whole((k, n), dtype, case + 1), whole((m, n), dtype, case + 2)
    b, res = whole((n,), F32, case + 3), whole((m, n), F32, case + 4)
    z = x.double() @ w.double() + b.double()
    want = (z.clamp(min=0) if act == "relu" else z) + res.double()
    out, pre = T.linear(x.cuda(), w.cuda(), b.cuda(), res.cuda(), act=act, out_dtype=F32, pre=True)
    assert torch.equal(out.cpu().double(), want)
    assert torch.equal(pre.cpu(), z.to(F32).to(dtype))
    pre = whole((m, n), dtype, case + 5)
    dz = torch.where(pre > 0, grad, 0).double() if act == "relu" else grad.double()
    for weight_dtype in (F32, dtype):
        dx, dw, db = T.linear_grad(grad.cuda(), x.cuda(), w.cuda(), pre.cuda(), act=act, weight_dtype=weight_dtype)
        assert torch.equal(dw.cpu(), (x.double().t() @ dz).to(F32).to(weight_dtype))
        assert torch.equal(dx.cpu(), (dz @ w.double().t()).to(F32).to(dtype))
        assert torch.equal(db.cpu().double(), dz.sum(0))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_act_at_any_argument(act, dtype):
    """Every size of argument, infinities and NaN, through a map that copies."""
    note(f"linear act {act} {dtype}")
    z = torch.cat([torch.linspace(-20, 20, 1021), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 100.0, -100.0, 3e4, -3e4])])
    x = z.to(dtype).view(-1, 1)
    one = torch.ones(1, 1, dtype=dtype)
    out, pre = T.linear(x.cuda(), one.cuda(), act=act, out_dtype=F32, pre=True)
    y, ty = act_of(x.double(), 2 * U * x.double().abs(), act)
    close(out, y, ty + 2.0 ** -120, F32, act)
    slope, ts = slope_of(x.double(), act)
    dx, _, _ = T.linear_grad(torch.ones_like(pre), x.cuda(), one.cuda(), pre, act=act)
    close(dx, slope, ts + 2 * U * slope.abs() + 2.0 ** -120 + (HALF[dtype] * slope.abs() if act != "none" else 0), dtype, act)
    far = torch.tensor([[math.inf], [-math.inf], [math.nan]]).to(dtype).cuda()
    got = T.linear(far, one.cuda(), act=act, out_dtype=F32).cpu().flatten()
    assert got[0] == math.inf and (got[1] == 0 if act != "none" else got[1] == -math.inf)
    assert got[2] == 0 if act == "relu" else torch.isnan(got[2])
    s = T.linear_grad(torch.ones_like(far), far, one.cuda(), far, act=act, need=("x",))[0].cpu().flatten()
    assert s[0] == 1 and s[1] == (1 if act == "none" else 0)


def test_linear_special_rows():
    """Infinities and NaN stay in the rows and columns they belong to, at every
    size's kernel."""
    note("linear special rows")
    for m, k, n in [(5, 100, 70), (300, 64, 72), (600, 520, 520), (2100, 264, 1032)]:
        for dtype in DTYPES:
            x, w = torch.ones(m, k, dtype=dtype), torch.ones(k, n, dtype=dtype)
            x[1, 0], x[m - 1, k - 1], w[3, n - 1] = math.inf, math.nan, -math.inf
            out = T.linear(x.cuda(), w.cuda(), out_dtype=F32).cpu()
            rest = torch.ones(m, dtype=torch.bool)
            rest[1] = rest[m - 1] = False
            assert (out[rest][:, :n - 1] == k).all() and (out[rest][:, n - 1] == -math.inf).all()
            assert (out[1, :n - 1] == math.inf).all() and torch.isnan(out[1, n - 1])
            assert torch.isnan(out[m - 1]).all()


def test_linear_differences():
    """The gradients against differences of the forward call."""
    note("linear differences")
    m, k, n = 23, 20, 18
    x, w, b, g = normal((m, k), F32, 1), normal((k, n), F32, 2, 0.3), normal((n,), F32, 3), normal((m, n), F32, 4)
    for act in ACTS[2:]:
        loss = lambda x_, w_, b_: float((T.linear(x_.cuda(), w_.cuda(), b_.cuda(), act=act).double().cpu() * g.double()).sum())
        _, pre = T.linear(x.cuda(), w.cuda(), b.cuda(), act=act, pre=True)
        dx, dw, db = T.linear_grad(g.cuda(), x.cuda(), w.cuda(), pre, act=act)
        args, grads = [x, w, b], [dx, dw, db]
        for i in range(3):
            v = normal(args[i].shape, F32, 10 + i)
            h = 2.0 ** -8
            up, down = ([a + (h if j == i else 0) * v if j == i else a for j, a in enumerate(args)],
                        [a - (h if j == i else 0) * v if j == i else a for j, a in enumerate(args)])
            slope = (loss(*up) - loss(*down)) / (2 * h)
            want = float((grads[i].double().cpu() * v.double()).sum())
            # the third derivatives of the sum along v, and rounding of its m n terms
            bound = h * h * float(v.double().pow(2).sum()) * 10 + m * n * 60 * U / h
            assert abs(slope - want) <= bound, (act, i, slope, want, bound)


# ----------------------------------------------------------- residual norm --

DEPTH = 48  # additions a term passes: up to 16 in a lane, 6 over lanes, 16 over waves, and scaling


def norm_of(v, tv, norm, d):
    """(out, tolerance, mean, tolerance, rstd, relative tolerance) of a row norm
    of v known to tv."""
    kind, eps = norm.get("kind", "layer"), norm.get("eps", 1e-5)
    if kind == "layer":
        mu = v.mean(1, keepdim=True)
        em = DEPTH * U * v.abs().mean(1, keepdim=True) + tv.mean(1, keepdim=True)
    else:
        mu, em = torch.zeros(v.shape[0], 1).double(), torch.zeros(v.shape[0], 1).double()
    dev = v - mu
    et = em + tv + U * dev.abs()
    var = (dev * dev).mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    ev = DEPTH * U * var + (2 * dev.abs() * et + et * et).mean(1, keepdim=True)
    tr = 0.5 * ev * r * r + 4 * U
    hat = dev * r
    eh = r * et + hat.abs() * (tr + 3 * U)
    w = torch.ones(d).double() if norm.get("weight") is None else norm["weight"].double()
    b = torch.zeros(d).double() if norm.get("bias") is None else norm["bias"].double()
    out = hat * w + b
    return out, eh * w.abs() + 3 * U * ((hat * w).abs() + b.abs()), mu, em, r, tr


def gate_rows(gate, off, m, d):
    """The gate of every row, and which rows there are."""
    inside = torch.ones(m, dtype=torch.bool)
    if off is None:
        return (torch.ones(1, d).double() if gate is None else gate.double().view(1, d)).expand(m, d), inside
    rows = torch.ones(m, d).double()
    inside[:] = False
    for s in range(len(off) - 1):
        inside[off[s]:off[s + 1]] = True
        if gate is not None:
            rows[off[s]:off[s + 1]] = gate[s].double()
    return rows, inside


def check_resnorm(x, f, scale, gate, off, post, pre, xs=None, fs=None):
    m, d = f.shape
    xs, fs = cuda(x) if xs is None else xs, cuda(f) if fs is None else fs
    dev = lambda norm: None if norm is None else {k: v.cuda() if torch.is_tensor(v) else v for k, v in norm.items()}
    doff = None if off is None else torch.tensor(off).cuda()
    out = torch.full((m, d), 7.0, dtype=x.dtype, device="cuda")
    out_h = torch.full((m, d), 7.0, dtype=f.dtype, device="cuda") if pre is not None else None
    y, h, stats = T.residual_norm(xs, fs, scale=scale, gate=cuda(gate), off=doff, post=dev(post), pre=dev(pre), out=out,
                                  out_h=out_h, stats=True)
    assert y is out and (h is out_h)
    g, inside = gate_rows(gate, off, m, d)
    g = g * float(torch.tensor(scale, dtype=F32))
    p, tp = f.double(), torch.zeros(m, d).double()
    want = torch.zeros(m, 4).double()
    tol = torch.zeros(m, 4).double()
    if post is not None:
        p, tp, mu, em, r, tr = norm_of(p, tp, post, d)
        want[:, 0:1], want[:, 1:2], tol[:, 0:1], tol[:, 1:2] = mu, r, em, r * tr
    ref = x.double() + g * p
    ty = g.abs() * tp + 4 * U * ((g * p).abs() + x.double().abs())
    close(y.cpu()[inside], ref[inside], ty[inside], x.dtype, "y")
    if pre is not None:
        rh, th, mu, em, r, tr = norm_of(ref, ty, pre, d)
        want[:, 2:3], want[:, 3:4], tol[:, 2:3], tol[:, 3:4] = mu, r, em, r * tr
        close(h.cpu()[inside], rh[inside], th[inside], f.dtype, "h")
        assert (h.cpu()[~inside] == 7.0).all()
    close(stats.cpu()[inside], want[inside], tol[inside], F32, "stats")
    assert (y.cpu()[~inside] == 7.0).all()
    return y, h, stats


def check_resnorm_grad(x, f, scale, gate, off, post, pre, y, stats, gy, gh, strides=None):
    m, d = f.shape
    lay = (lambda t: cuda(t)) if strides is None else (lambda t: None if t is None else strided(t, *strides))
    dev = lambda norm: None if norm is None else {k: v.cuda() if torch.is_tensor(v) else v for k, v in norm.items()}
    args = (lay(gy), lay(gh), lay(y), lay(f), stats.cuda() if post is not None or pre is not None else None)
    kw = dict(scale=scale, gate=cuda(gate), off=None if off is None else torch.tensor(off).cuda(), post=dev(post), pre=dev(pre))
    got = T.residual_norm_grad(*args, **kw)
    rows, inside = gate_rows(gate, off, m, d)
    # rows outside count for nothing: everything of theirs is taken as zero
    take = lambda t: torch.where(inside.unsqueeze(1), t.double(), 0.0)
    s32 = float(torch.tensor(scale, dtype=F32))
    st = take(stats.cpu())
    dy = torch.zeros(m, d).double() if gy is None else take(gy)
    ty = torch.zeros(m, d).double()
    sums = {}

    def add(name, terms, errors):
        sums[name] = (terms.sum(0), errors.sum(0) + m * U * (terms.abs() + errors).sum(0))

    def back(g, tg, hat, r, kind):
        """The gradient of a row norm; its tolerance to first order."""
        gh_ = g * hat
        c2, t2 = gh_.mean(1, keepdim=True), (tg * hat.abs() + 4 * U * gh_.abs()).mean(1, keepdim=True) + DEPTH * U * gh_.abs().mean(1, keepdim=True)
        c1, t1 = torch.zeros(m, 1).double(), torch.zeros(m, 1).double()
        if kind == "layer":
            c1, t1 = g.mean(1, keepdim=True), tg.mean(1, keepdim=True) + DEPTH * U * g.abs().mean(1, keepdim=True)
        v = r * (g - c1 - hat * c2)
        return v, r * (tg + t1 + hat.abs() * t2 + 6 * U * (g.abs() + c1.abs() + 2 * (hat * c2).abs()))

    if pre is not None:
        r = st[:, 3:4]
        hat = take((y.double().cpu() - st[:, 2:3])) * r
        g = take(gh)
        add("pre_weight", g * hat, 5 * U * (g * hat).abs())
        add("pre_bias", g, 0 * g)
        w = torch.ones(d).double() if pre.get("weight") is None else pre["weight"].double()
        v, t = back(g * w, 2 * U * (g * w).abs(), hat, r, pre.get("kind", "layer"))
        dy, ty = dy + v, t + 2 * U * (dy.abs() + v.abs())
    if gy is not None or pre is not None:
        close(got.x.cpu()[inside], dy[inside], ty[inside], y.dtype, "dx")
    p, tp, hat1, r = take(f), torch.zeros(m, d).double(), None, None
    w1 = torch.ones(d).double()
    if post is not None:
        r = st[:, 1:2]
        hat1 = (take(f) - st[:, 0:1]) * r
        w1 = w1 if post.get("weight") is None else post["weight"].double()
        b1 = torch.zeros(d).double() if post.get("bias") is None else post["bias"].double()
        p, tp = take(hat1 * w1 + b1), 5 * U * ((hat1 * w1).abs() + b1.abs())
    sd, tsd = s32 * dy, abs(s32) * ty + U * (s32 * dy).abs()
    each, terr = sd * p, tsd * p.abs() + sd.abs() * tp + 2 * U * (sd * p).abs()
    if gate is not None and off is None:
        add("gate", each, terr)
    elif gate is not None:
        n = len(off) - 1
        tot, tt = torch.zeros(n, d).double(), torch.zeros(n, d).double()
        for i in range(n):
            e = slice(off[i], off[i + 1])
            tot[i] = each[e].sum(0)
            tt[i] = terr[e].sum(0) + (off[i + 1] - off[i]) * U * (each[e].abs() + terr[e]).sum(0)
        sums["gate"] = (tot, tt)
    dp, tdp = sd * rows, tsd * rows.abs() + 2 * U * (sd * rows).abs()
    df, tdf = dp, tdp
    if post is not None:
        add("post_weight", dp * hat1, tdp * hat1.abs() + 5 * U * (dp * hat1).abs())
        add("post_bias", dp, tdp)
        g = dp * w1
        df, tdf = back(g, tdp * w1.abs() + 4 * U * g.abs(), hat1, r, post.get("kind", "layer"))
    close(got.f.cpu()[inside], df[inside], tdf[inside], f.dtype, "df")
    given = dict(gate=gate is not None, post_weight=post is not None and post.get("weight") is not None,
                 post_bias=post is not None and post.get("bias") is not None,
                 pre_weight=pre is not None and pre.get("weight") is not None,
                 pre_bias=pre is not None and pre.get("bias") is not None)
    for name, there in given.items():
        t = getattr(got, name)
        assert (t is not None) == there
        if there:
            close(t, *sums[name], F32, name)
    for need in (("x",), ("f", "post"), ("gate", "pre")):
        part = T.residual_norm_grad(*args, **kw, need=need)
        for name, t in zip(part._fields, part):
            full = getattr(got, name)
            asked = name.split("_")[0] in need
            assert (t is None) == (full is None or not asked)
            if t is not None and name in ("x", "f"):
                assert torch.equal(t[inside.cuda()], full[inside.cuda()])
            elif t is not None:
                assert torch.equal(t, full)


RESNORM = [  # rows, channels, segments' sizes or None, rows before the first
    (1, 1, None), (5, 3, None), (7, 8, None), (33, 47, None), (1, 4096, None), (9, 128, None), (300, 64, None),
    (65, 172, None), (50, 500, None), (41, 512, None), (20, 520, None), (6, 1001, None), (11, 2048, None),
    (3, 2056, None), (4, 5000, None), (2, 8192, None), (3, 4100, None), (5000, 16, None), (1003, 200, None),
    (64, 40, [10, 0, 1, 53]), (300, 128, [0, 0, 300, 0]), (100, 33, [1] * 100), (500, 96, [200, 3, 0, 250]),
    (90, 600, [31, 0, 40]), (40, 4200, [7, 1, 0, 20]), (0, 24, None), (0, 24, [0, 0]), (700, 12, [690]), (20, 64, []),
    (3000, 24, [1500, 2, 1400]), (2000, 700, [1990]),
]
NORMS = [None, "layer", "rms"]


def make_norm(kind, d, seed, weight=True, bias=True):
    if kind is None:
        return None
    return dict(kind=kind, weight=1 + normal((d,), F32, seed, 0.3) if weight else None,
                bias=normal((d,), F32, seed + 1, 0.3) if bias else None, eps=[1e-5, 1e-3][seed % 2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(RESNORM)))
def test_residual_norm(dtype, case):
    m, d, sizes = RESNORM[case]
    off = None if sizes is None else ranges(sizes, lead=min(3, m - sum(sizes))).tolist()
    for i in range(3):
        stream = F32 if (case + i) % 3 == 0 else dtype
        post = make_norm(NORMS[(case + i) % 3], d, case, (case + i) % 4 != 1, (case + i) % 2 == 0)
        pre = make_norm(NORMS[(case // 3 + 2 * i + 1) % 3], d, case + 7, (case + i) % 5 != 2, (case + i) % 2 == 1)
        gate = None
        if (case + i) % 4:
            gate = normal((d,) if off is None else (len(off) - 1, d), F32, case + 9)
        note(f"residual_norm {dtype} stream {stream} m={m} d={d} segments={sizes and len(sizes)} post={post and post['kind']} "
             f"pre={pre and pre['kind']} gate={gate is not None}")
        x = normal((m, d), stream, case + 1, 2.0) + normal((d,), stream, case + 2)
        f = normal((m, d), dtype, case + 3) + normal((d,), dtype, case + 4, 0.5)
        y, h, stats = check_resnorm(x, f, 0.7, gate, off, post, pre)
        gy = normal((m, d), stream, case + 5) if (case + i) % 5 else None
        gh = normal((m, d), dtype, case + 6) if pre is not None else None
        _, inside = gate_rows(None, off, m, d)
        y = torch.where(inside.unsqueeze(1), y.cpu(), 1.0).to(stream)
        stats = torch.where(inside.unsqueeze(1), stats.cpu(), 1.0)
        check_resnorm_grad(x, f, 0.7, gate, off, post, pre, y, stats, gy, gh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,pad,lead", [(16, 8, 0), (16, 3, 1), (12, 4, 4), (5, 1, 2), (130, 2, 1), (700, 5, 3), (4101, 3, 0)])
def test_residual_norm_strided(dtype, d, pad, lead):
    note(f"residual_norm strided {dtype} d={d} pad={pad} lead={lead}")
    m = 37
    x, f = normal((m, d), dtype, 1, 2.0), normal((m, d), dtype, 2)
    post, pre, gate = make_norm("rms", d, 3), make_norm("layer", d, 5), normal((d,), F32, 7)
    y, h, stats = check_resnorm(x, f, 1.3, gate, None, post, pre, strided(x, pad, lead), strided(f, pad, lead))
    wide, wide_h = (torch.full((m, lead + d + pad), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    dev = lambda norm: {k: v.cuda() if torch.is_tensor(v) else v for k, v in norm.items()}
    T.residual_norm(x.cuda(), f.cuda(), scale=1.3, gate=gate.cuda(), post=dev(post), pre=dev(pre),
                    out=wide[:, lead:lead + d], out_h=wide_h[:, lead:lead + d])
    assert torch.equal(wide[:, lead:lead + d], y) and torch.equal(wide_h[:, lead:lead + d], h)
    for t in (wide, wide_h):
        assert (torch.cat([t[:, :lead], t[:, lead + d:]], 1) == 7.0).all()
    check_resnorm_grad(x, f, 1.3, gate, None, post, pre, y.cpu(), stats.cpu(), normal((m, d), dtype, 8),
                       normal((m, d), dtype, 9), (pad, lead))


COUNTED_ROWS = [  # rows, channels, segments (None: one gate for all): many rows a worker, segments within one and over
    # several workers, teams of lanes and of all waves
    (300_001, 128, 9000), (100_003, 24, None), (200_001, 8, 40), (33_000, 512, None), (33_001, 520, 3), (20_000, 600, 300),
    (5000, 4096, 5), (3001, 8192, None), (70_007, 3, 2000), (9001, 2050, 9000),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(COUNTED_ROWS)))
def test_residual_norm_sums_are_exact(dtype, case):
    """The sums over rows on whole numbers, which fp32 holds exactly however they
    are added (at most 24 a row, 300,001 rows: below 2^24): the statistics given
    are whole, and the norm before has weights of 0, so that what comes back
    through it is 0 and its own sums are whole too."""
    m, d, segments = COUNTED_ROWS[case]
    stream = [dtype, F32][case % 2]
    note(f"residual_norm sums {dtype} stream {stream} m={m} d={d} segments={segments}")
    f, y = whole((m, d), dtype, case), whole((m, d), stream, case + 1)
    gy, gh = whole((m, d), stream, case + 2).sign(), whole((m, d), dtype, case + 3).sign()
    g = torch.Generator().manual_seed(case + 4)
    stats = torch.stack([torch.randint(-1, 2, (m,), generator=g), torch.randint(1, 3, (m,), generator=g)] * 2, 1).float()
    off = None
    if segments is not None:
        off = torch.cat([torch.zeros(1), torch.randint(0, m + 1, (segments - 1,), generator=g).sort().values, torch.tensor([m])]).long()
    gate = whole((d,) if off is None else (segments, d), F32, case + 5)
    w, b, zero = whole((d,), F32, case + 6), whole((d,), F32, case + 7), torch.zeros(d)
    got = T.residual_norm_grad(gy.cuda(), gh.cuda(), y.cuda(), f.cuda(), stats.cuda(), gate=gate.cuda(),
                               off=None if off is None else off.cuda(), post=dict(kind="rms", weight=w.cuda(), bias=b.cuda()),
                               pre=dict(kind="layer", weight=zero.cuda(), bias=zero.cuda()))
    hat1 = (f.float() - stats[:, 0:1]) * stats[:, 1:2]
    hat2 = (y.float() - stats[:, 2:3]) * stats[:, 3:4]
    gy, gh = gy.float(), gh.float()
    assert torch.equal(got.x.float().cpu(), gy)
    each, terms = gy * (w * hat1 + b), gy * hat1
    if off is None:
        dgate, rows = each.double().sum(0), gate.expand(m, d)
    else:
        seg = torch.searchsorted(off, torch.arange(m), right=True) - 1
        dgate, rows = torch.zeros(segments, d, dtype=torch.float64).index_add_(0, seg, each.double()), gate[seg]
    for got_sum, want in ((got.gate, dgate), (got.post_weight, (rows * terms).double().sum(0)),
                          (got.post_bias, (rows * gy).double().sum(0)), (got.pre_weight, (gh * hat2).double().sum(0)),
                          (got.pre_bias, gh.double().sum(0))):
        assert float(want.abs().max()) < 2 ** 24
        assert torch.equal(got_sum.cpu().double(), want)


def test_residual_norm_special_rows():
    """Constant rows, rows far from zero, infinities and NaN: each keeps to
    itself."""
    note("residual_norm special rows")
    for d in (40, 1030):
        f = normal((8, d), F32, 1)
        f[1], f[2], f[3, 5], f[4, d - 1] = 3.0, 1e6 + torch.arange(d) % 2, math.inf, math.nan
        x = torch.zeros(8, d)
        for kind in ("layer", "rms"):
            y, h = T.residual_norm(x.cuda(), f.cuda(), post=dict(kind=kind), pre=dict(kind=kind))
            clean = T.residual_norm(x[[0, 5, 6, 7]].cuda(), f[[0, 5, 6, 7]].cuda(), post=dict(kind=kind), pre=dict(kind=kind))
            assert torch.equal(y[[0, 5, 6, 7]], clean[0]) and torch.equal(h[[0, 5, 6, 7]], clean[1])
            assert (y[1] == 0).all() if kind == "layer" else (y[1] - 1).abs().max() < 1e-5
            want, tol = norm_of(f[2:3].double(), torch.zeros(1, d).double(), dict(kind=kind), d)[:2]
            close(y[2:3], want, tol, F32, "far from zero")
            assert torch.isnan(y[3]).any() and torch.isnan(y[4]).all() and torch.isnan(h[3]).all()


def test_residual_norm_differences():
    note("residual_norm differences")
    m, d, off = 12, 20, [0, 5, 5, 12]
    x, f, gate = normal((m, d), F32, 1), normal((m, d), F32, 2), normal((3, d), F32, 3)
    gy, gh = normal((m, d), F32, 4), normal((m, d), F32, 5)
    doff = torch.tensor(off).cuda()
    for kinds in (("layer", "rms"), ("rms", "layer")):
        pw, pb, qw, qb = (normal((d,), F32, 6 + i, 0.3) + (1 - i % 2) for i in range(4))

        def call(x, f, gate, pw, pb, qw, qb, stats=False):
            return T.residual_norm(x.cuda(), f.cuda(), scale=0.9, gate=gate.cuda(), off=doff,
                                   post=dict(kind=kinds[0], weight=pw.cuda(), bias=pb.cuda()),
                                   pre=dict(kind=kinds[1], weight=qw.cuda(), bias=qb.cuda()), stats=stats)

        def loss(*args):
            y, h = call(*args)
            return float((y.double().cpu() * gy.double()).sum() + (h.double().cpu() * gh.double()).sum())

        args = [x, f, gate, pw, pb, qw, qb]
        y, h, stats = call(*args, stats=True)
        grads = T.residual_norm_grad(gy.cuda(), gh.cuda(), y, f.cuda(), stats, scale=0.9, gate=gate.cuda(), off=doff,
                                     post=dict(kind=kinds[0], weight=pw.cuda(), bias=pb.cuda()),
                                     pre=dict(kind=kinds[1], weight=qw.cuda(), bias=qb.cuda()))
        for i, g in enumerate(grads):
            v = normal(args[i].shape, F32, 20 + i)
            hstep = 2.0 ** -8
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + hstep * v, args[i] - hstep * v
            slope = (loss(*up) - loss(*down)) / (2 * hstep)
            want = float((g.double().cpu() * v.double()).sum())
            bound = hstep * hstep * float(v.double().pow(2).sum()) * 60 + 2 * m * d * 100 * U / hstep
            assert abs(slope - want) <= bound, (kinds, i, slope, want, bound)


# --------------------------------------------------------- label log probs --

def labels_reference(x, labels, scale):
    """(logp, stats, entropy, all log probabilities) and tolerances, in 64 bits."""
    m, c = x.shape
    l = x.double() * float(torch.tensor(scale, dtype=F32))
    live = l > -math.inf
    most = l.max(1, keepdim=True).values
    none = ~live.any(1, keepdim=True)
    ref = torch.where(none, 0.0, most)
    e = torch.exp(l - ref)
    S = e.sum(1, keepdim=True)
    log_s = torch.where(none, 0.0, torch.log(S))
    lp = torch.where(live, l - ref - log_s, -math.inf)
    dist = torch.where(live, ref - l, 0.0)
    H = torch.where(none, 0.0, log_s + (e * dist).sum(1, keepdim=True) / torch.where(none, 1.0, S))
    # scaling and subtracting round to u of their sizes, which the exponential
    # makes relative (its own error is 4 u); a lane adds up to c / 64 terms, and
    # a new maximum rescales by 8 u, at most once a step
    size = torch.where(live, l.abs(), 0.0)
    a = 3 * U * size.max(1, keepdim=True).values
    ts = a + (3 * c / 64 + 96) * U
    tlp = ts + a + 3 * U * (log_s.abs() + torch.where(live, lp.abs(), 0.0))
    th = ts * (3 + 3 * (H - log_s).abs()) + a + 4 * U * (H.abs() + log_s.abs())
    return lp, tlp, torch.cat([most, log_s], 1), torch.cat([a, ts + 2 * U * log_s.abs()], 1), H, th


def close_special(got, ref, tol, dtype, what):
    """close, with equal infinities."""
    got, fine = got.double().cpu(), torch.isfinite(ref)
    assert torch.equal(got[~fine], ref[~fine]), what
    close(got[fine], ref[fine], tol.expand_as(ref)[fine], dtype, what)


def check_labels(x, labels, scale, top, xs=None):
    m, c = x.shape
    r = T.label_log_probs(cuda(x) if xs is None else xs, cuda(labels), scale, top=top, entropy=True)
    lp, tlp, stats, tstats, H, th = labels_reference(x, labels, scale)
    known = (labels >= 0) & (labels < c)
    at = torch.where(known, labels, 0).long().unsqueeze(1)
    want = torch.where(known, lp.gather(1, at).squeeze(1), 0.0)
    close_special(r.logp, want, torch.where(known, tlp.gather(1, at).squeeze(1), 0.0), F32, "logp")
    close_special(r.stats, stats, tstats, F32, "stats")
    close(r.entropy, H.squeeze(1), th.squeeze(1), F32, "entropy")
    if not top:
        assert r.top_ids is None and r.top_logp is None
        return r
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :top]
    v = lp.gather(1, order)
    ids = torch.where(v > -math.inf, order, -1)
    assert torch.equal(r.top_ids.cpu().long(), ids), (r.top_ids.cpu().long() != ids).nonzero()[:4]
    close_special(r.top_logp, v, tlp.gather(1, order), F32, "top_logp")
    return r


def check_labels_grad(x, labels, scale, r, g, h, xs=None):
    m, c = x.shape
    dx = T.label_log_probs_grad(cuda(x) if xs is None else xs, cuda(labels), r.stats, cuda(g), scale,
                                entropy=None if h is None else r.entropy, grad_entropy=cuda(h))
    s32 = float(torch.tensor(scale, dtype=F32))
    l = x.double() * s32
    st, H = r.stats.double().cpu(), r.entropy.double().cpu().unsqueeze(1)
    none = st[:, :1] == -math.inf
    live = l > -math.inf
    lp = torch.where(live, l - torch.where(none, 0.0, st[:, :1]) - st[:, 1:], -math.inf)
    p = torch.where(none, 0.0, torch.exp(lp))
    lp0 = torch.where(live, lp, 0.0)
    tl = 3 * U * (torch.where(live, l.abs(), 0.0) + torch.where(none, 0.0, st[:, :1]).abs() + st[:, 1:].abs() + lp0.abs())
    known = (labels >= 0) & (labels < c) if labels is not None else torch.zeros(m, dtype=torch.bool)
    gg = torch.where(known, g.double() if g is not None else torch.zeros(m).double(), 0.0).unsqueeze(1)
    hh = torch.zeros(m, 1).double() if h is None else h.double().unsqueeze(1)
    one = torch.zeros(m, c).double()
    if labels is not None:
        one.scatter_(1, torch.where(known, labels, 0).long().unsqueeze(1), known.double().unsqueeze(1))
    spread = torch.where(live, lp0 + H, 0.0)
    want = torch.where(none, 0.0, s32 * (gg * (one - p) - hh * p * spread))
    tol = abs(s32) * (gg.abs() * (p * (tl + 8 * U) + 2 * U * one) +
                      hh.abs() * p * (spread.abs() * (tl + 8 * U) + tl + 2 * U * (lp0.abs() + H.abs()))) + 2.0 ** -120
    tol = tol + 2 * U * want.abs()
    close(dx, want, tol, x.dtype, "dx")
    return dx


LABELS = [  # rows, classes, alternatives
    (1, 1, 1), (5, 2, 2), (9, 3, 0), (77, 11, 4), (33, 96, 8), (50, 700, 20), (300, 47, 5), (64, 64, 64), (1000, 172, 3), (7, 1000, 20), (50, 1024, 64),
    (3, 1025, 1), (40, 1500, 10), (2100, 1100, 4), (5, 40_003, 64), (2, 300_001, 20), (130, 5000, 8), (1200, 2050, 0),
    (0, 9, 2), (2500, 17, 17), (1, 70_000, 50),
]


def logits(m, c, dtype, seed, masked):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, c), generator=g) * 3 + torch.randn((c,), generator=g)
    if masked and c > 1:
        x[torch.rand((m, c), generator=g) < 0.1] = -math.inf
        if m > 2:
            x[1] = -math.inf
            x[2] = -math.inf
            x[2, c // 2] = 0.5
    return x.to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LABELS)))
def test_label_log_probs(dtype, case):
    m, c, top = LABELS[case]
    g = torch.Generator().manual_seed(case)
    labels = torch.randint(0, c, (m,), generator=g, dtype=torch.int32)
    if m > 3:
        labels[0], labels[3] = -1, c
    for masked in (False, True):
        scale = [1.0, 0.7, 2.5][(case + masked) % 3]
        note(f"label_log_probs {dtype} m={m} c={c} top={top} masked={masked}")
        x = logits(m, c, dtype, case + 50 * masked, masked)
        r = check_labels(x, labels, scale, top)
        gl, gh = normal((m,), F32, case + 1), normal((m,), F32, case + 2)
        check_labels_grad(x, labels, scale, r, gl, gh if (case + masked) % 2 else None)
        check_labels_grad(x, None, scale, r, None, gh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("c,pad,lead", [(16, 8, 0), (47, 3, 1), (5, 1, 2), (1100, 5, 3), (9000, 7, 1)])
def test_label_log_probs_strided(dtype, c, pad, lead):
    note(f"label_log_probs strided {dtype} c={c} pad={pad} lead={lead}")
    m = 21
    x = logits(m, c, dtype, c, True)
    labels = torch.randint(0, c, (m,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    xs = strided(x, pad, lead)
    r = check_labels(x, labels, 1.0, min(c, 7), xs)
    dx = check_labels_grad(x, labels, 1.0, r, normal((m,), F32, 1), normal((m,), F32, 2), xs)
    wide = torch.full((m, lead + c + pad), 7.0, dtype=dtype, device="cuda")
    T.label_log_probs_grad(xs, labels.cuda(), r.stats, normal((m,), F32, 1).cuda(), entropy=r.entropy,
                           grad_entropy=normal((m,), F32, 2).cuda(), out=wide[:, lead:lead + c])
    assert torch.equal(wide[:, lead:lead + c], dx)
    assert (torch.cat([wide[:, :lead], wide[:, lead + c:]], 1) == 7.0).all()


@pytest.mark.parametrize("c", [12, 600, 3000, 50_000])
def test_label_log_probs_ties(c):
    """Equal logits, zeros of both signs among them: the lower class first."""
    note(f"label_log_probs ties c={c}")
    m, top = 6, min(c, 64)
    x = torch.zeros(m, c)
    x[1, ::2] = -0.0
    x[2] = (torch.arange(c) % 3).float()
    x[3] = -(torch.arange(c) // 5 % 7).float()
    x[4, c - 3:] = 1.0
    x[5] = torch.arange(c).float() / 64
    labels = torch.arange(m, dtype=torch.int32)
    for dtype in DTYPES:
        check_labels(x.to(dtype), labels, 1.0, top)


@pytest.mark.parametrize("c", [5, 500, 3000, 30_000])
@pytest.mark.parametrize("m", [7, 3000])
def test_label_log_probs_special_rows(m, c):
    """NaN and +inf mark their row and no other."""
    note(f"label_log_probs special rows m={m} c={c}")
    x = logits(7, c, F32, 3, False).repeat((m + 6) // 7, 1)[:m].contiguous()
    x[1, c - 1], x[3, 2], x[4, 1], x[4, 0] = math.nan, math.inf, math.inf, -math.inf
    labels = torch.full((m,), 2, dtype=torch.int32)
    clean = [i for i in range(m) if i not in (1, 3, 4)]
    r = T.label_log_probs(x.cuda(), labels.cuda(), top=3, entropy=True)
    ref = T.label_log_probs(logits(7, c, F32, 3, False).repeat((m + 6) // 7, 1)[:m].contiguous().cuda(), labels.cuda(), top=3,
                            entropy=True)
    for a, b in zip(r, ref):
        assert torch.equal(a[clean], b[clean])
    for i in (1, 3, 4):
        assert torch.isnan(r.logp[i]) and torch.isnan(r.entropy[i]) and torch.isnan(r.stats[i]).all()
        assert torch.isnan(r.top_logp[i]).all() and (r.top_ids[i] == -1).all()
    dx = T.label_log_probs_grad(x.cuda(), labels.cuda(), r.stats, torch.ones(m).cuda())
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[clean]).all()


@pytest.mark.parametrize("c", [40, 2000])
def test_label_log_probs_of_any_size(c):
    """Logits far from zero, and classes that all but one are far below."""
    note(f"label_log_probs sizes c={c}")
    x = logits(6, c, F32, 9, False)
    x[0] += 1e4
    x[1] -= 1e4
    x[2] *= 1e4
    x[3], x[3, 7] = -1e30, 5.0
    x[4] = -3e38
    x[5] *= 1e-30
    labels = torch.full((6,), 7, dtype=torch.int32)
    r = check_labels(x, labels, 1.0, 5)
    check_labels_grad(x, labels, 1.0, r, normal((6,), F32, 1), normal((6,), F32, 2))
    # scaled past the range: the row of -3e38 is masked, one of 3e38 infinite
    r = T.label_log_probs(x[4:5].cuda(), labels[:1].cuda(), 4.0, top=2, entropy=True)
    assert r.logp[0] == -math.inf and r.entropy[0] == 0 and (r.top_ids == -1).all() and (r.top_logp == -math.inf).all()
    assert torch.isnan(T.label_log_probs(-x[4:5].cuda(), labels[:1].cuda(), 4.0).logp[0])


COUNTED = [  # rows, classes: of every form, in parts and not, with and without a rest of a vector
    (300, 47), (70, 172), (9, 1000), (40, 1024), (3, 1025), (2100, 1100), (1200, 2050), (130, 5000), (5, 40_003),
    (2, 300_001), (1, 70_000), (1030, 20_001), (3, 300_000),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(COUNTED)))
def test_label_log_probs_counts_every_class(dtype, case):
    """Rows whose live classes all have a logit of 0, the others -inf: S is their
    number, which fp32 holds exactly however it is added, so that a class lost
    or counted twice moves log S by 1 / S, against 6 u of log S.  The live ones
    of a row: all (a lost vector moves log S by 8 / c); the last vector's; the
    first's; a wave's length around every multiple of 1,024 and around the
    borders of parts; every second."""
    m, c = COUNTED[case]
    note(f"label_log_probs counted {dtype} m={m} c={c}")
    e = min(c, 4 if dtype == F32 else 8)
    j = torch.arange(c)
    parts = max(1, min(1024 // m, c // 2048))
    per = -(-(-(-c // e)) // parts) * e  # classes of a part
    near = lambda p: ((j + 3) % p < 6) & (j > 3)
    masks = [torch.ones(c, dtype=torch.bool), j >= c - e, j < e, near(1024) | (j == c - 1), near(per) | (j == 0), j % 2 == 1]
    for first in range(0, len(masks), m):
        live = torch.stack([masks[(first + r) % len(masks)] for r in range(m)])
        x = torch.where(live, 0.0, -math.inf).to(dtype)
        labels = torch.tensor([int(v.nonzero()[-1]) for v in masks], dtype=torch.int32)[(first + torch.arange(m)) % len(masks)]
        r = T.label_log_probs(x.cuda(), labels.cuda(), 1.0, top=min(c, 3), entropy=True)
        log_s = live.sum(1).double().log()
        close(r.stats, torch.stack([torch.zeros(m).double(), log_s], 1), 6 * U * torch.stack([log_s, log_s], 1), F32, "stats")
        close(r.logp, -log_s, 6 * U * log_s, F32, "logp")
        close(r.entropy, log_s, 6 * U * log_s, F32, "entropy")
        firsts = torch.stack([torch.nn.functional.pad(v.nonzero().flatten()[:min(c, 3)].int(), (0, max(0, min(c, 3) - int(v.sum()))),
                                                      value=-1) for v in masks])
        assert torch.equal(r.top_ids.cpu(), firsts[(first + torch.arange(m)) % len(masks)])


def test_label_log_probs_differences():
    note("label_log_probs differences")
    m, c = 6, 30
    x = logits(m, c, F32, 2, False)
    labels = torch.tensor([3, -1, 29, 0, 7, 7], dtype=torch.int32)
    g, h, v = normal((m,), F32, 3), normal((m,), F32, 4), normal((m, c), F32, 5)

    def loss(x_):
        r = T.label_log_probs(x_.cuda(), labels.cuda(), 0.8, entropy=True)
        return float((r.logp.double().cpu() * g.double()).sum() + (r.entropy.double().cpu() * h.double()).sum())

    r = T.label_log_probs(x.cuda(), labels.cuda(), 0.8, entropy=True)
    dx = T.label_log_probs_grad(x.cuda(), labels.cuda(), r.stats, g.cuda(), 0.8, entropy=r.entropy, grad_entropy=h.cuda())
    step = 2.0 ** -7
    slope = (loss(x + step * v) - loss(x - step * v)) / (2 * step)
    want = float((dx.double().cpu() * v.double()).sum())
    bound = step * step * float(v.double().abs().pow(3).sum()) * 4 + 2 * m * 200 * U / step
    assert abs(slope - want) <= bound, (slope, want, bound)


# ---------------------------------------------------------------- together --

def everything(t):
    """One training step's passes over the tensors of `t`: a block and a
    classifier, forward and back."""
    norm = lambda kind, name: dict(kind=kind, weight=t[name + "_w"], bias=t[name + "_b"])
    post, pre = norm("rms", "post"), norm("layer", "pre")
    f, z = T.linear(t["x"], t["w1"], t["b1"], act="gelu", pre=True)
    y, h, st = T.residual_norm(t["x"], f, scale=0.8, gate=t["gate"], off=t["off"], post=post, pre=pre, stats=True)
    logits = T.linear(h, t["w2"], t["b2"], t["res"], out_dtype=h.dtype)
    r = T.label_log_probs(logits, t["labels"], 0.9, top=4, entropy=True)
    dl = T.label_log_probs_grad(logits, t["labels"], r.stats, t["g"], 0.9, entropy=r.entropy, grad_entropy=t["g"])
    dh, dw2, db2 = T.linear_grad(dl, h, t["w2"])
    d = T.residual_norm_grad(t["gy"], dh, y, f, st, scale=0.8, gate=t["gate"], off=t["off"], post=post, pre=pre)
    dx, dw1, db1 = T.linear_grad(d.f, t["x"], t["w1"], z, act="gelu")
    return [f, z, y, h, st, logits, *r, dl, dh, dw2, db2, *d, dx, dw1, db1]


def everything_inputs(seed, dtype=BF16, m=3000, d=64, c=1200):
    off = ranges([m // 2, 0, 40, m - m // 2 - 40])
    labels = torch.randint(-1, c, (m,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    t = dict(x=normal((m, d), dtype, seed), w1=normal((d, d), dtype, seed + 1, 0.2), b1=normal((d,), F32, seed + 2),
             gate=normal((4, d), F32, seed + 3), off=off, post_w=normal((d,), F32, seed + 4), post_b=normal((d,), F32, seed + 5),
             pre_w=normal((d,), F32, seed + 6), pre_b=normal((d,), F32, seed + 7), w2=normal((d, c), dtype, seed + 8, 0.2),
             b2=normal((c,), F32, seed + 9), res=normal((m, c), dtype, seed + 10), labels=labels, g=normal((m,), F32, seed + 11),
             gy=normal((m, d), dtype, seed + 12))
    return {k: v.cuda() for k, v in t.items()}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c", [(3000, 1200), (9, 40_000)])
def test_graph_replays(dtype, m, c):
    """A captured pass replays with new inputs, between eager work; two graphs'
    workspaces are their own."""
    note(f"graph {dtype} m={m} c={c}")
    make = lambda seed: everything_inputs(seed, dtype, m, c=c) if m > 100 else dict(
        everything_inputs(seed, dtype, m, c=c), off=ranges([m // 2, 0, 1, m - m // 2 - 1]).cuda())
    t = make(1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        everything(t)
    torch.cuda.current_stream().wait_stream(s)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(t)
    with torch.cuda.graph(second):
        outs2 = everything(t)
    for seed in (1, 2, 3, 4):
        for key, v in make(seed).items():
            t[key].copy_(v)
        want = everything(t)
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        for i, (a, b, c_) in enumerate(zip(outs, outs2, want)):
            assert torch.equal(a, c_) and torch.equal(b, c_), (seed, i)


@pytest.mark.parametrize("dtype", DTYPES)
def test_results_repeat_whatever_memory_held(dtype):
    """The same bits again, with workspaces and outputs in memory that held NaN
    (large products and cut ones, sums joined over workgroups, long label rows)."""
    note(f"repeats {dtype}")
    t, u = everything_inputs(1, dtype), everything_inputs(2, dtype, m=9, c=40_000)
    u["off"] = ranges([4, 0, 1, 4]).cuda()
    m, k, n = 16_500, 264, 1480
    x, w, g, z = (normal(s, dtype, 3 + i).cuda() for i, s in enumerate([(m, k), (k, n), (m, n), (m, n)]))

    def run():
        return [*everything(t), *everything(u), T.linear(x, w, act="silu"), *T.linear_grad(g, x, w, z, act="gelu")]
    want = run()
    for _ in range(3):
        junk = [torch.full((1 << s,), math.nan, device="cuda") for s in range(10, 26)]
        del junk  # what is made next lies there
        for i, (a, b) in enumerate(zip(run(), want)):
            assert a is None and b is None or torch.equal(a, b), i


def test_streams():
    """Two streams at once, and the stream argument, give the eager bits."""
    note("streams")
    t, u = everything_inputs(1), everything_inputs(2, m=11_000)
    want, want2 = everything(t), everything(u)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            got = everything(t)
        with torch.cuda.stream(b):
            got2 = everything(u)
        torch.cuda.synchronize()
        for x, y in zip(got + got2, want + want2):
            assert torch.equal(x, y)
    f, z = T.linear(t["x"], t["w1"], t["b1"], act="gelu", pre=True, stream=a)
    norms = dict(post=dict(kind="rms", weight=t["post_w"], bias=t["post_b"]),
                 pre=dict(kind="layer", weight=t["pre_w"], bias=t["pre_b"]))
    y, h, st = T.residual_norm(t["x"], f, scale=0.8, gate=t["gate"], off=t["off"], stats=True, stream=a, **norms)
    logits = T.linear(h, t["w2"], t["b2"], t["res"], stream=a)
    r = T.label_log_probs(logits, t["labels"], 0.9, top=4, entropy=True, stream=a)
    dl = T.label_log_probs_grad(logits, t["labels"], r.stats, t["g"], 0.9, entropy=r.entropy, grad_entropy=t["g"], stream=a)
    dh, dw2, db2 = T.linear_grad(dl, h, t["w2"], stream=a)
    d = T.residual_norm_grad(t["gy"], dh, y, f, st, scale=0.8, gate=t["gate"], off=t["off"], stream=a, **norms)
    dx, dw1, db1 = T.linear_grad(d.f, t["x"], t["w1"], z, act="gelu", stream=a)
    a.synchronize()
    for x, y in zip([f, z, y, h, st, logits, *r, dl, dh, dw2, db2, *d, dx, dw1, db1], want):
        assert torch.equal(x, y)


def test_far_rows():
    """Rows far apart in arrays of 2.6e9 values, past what 32 bits hold, give
    the dense rows' bits."""
    note("far rows")
    m, apart, k, n = 40_001, 65_600, 64, 72

    def far(t):
        out = torch.empty(m * apart, dtype=BF16, device="cuda").view(m, apart)[:, :t.shape[1]]
        out.copy_(t)
        return out
    x, dy, w = normal((m, k), BF16, 1).cuda(), normal((m, n), BF16, 2).cuda(), normal((k, n), BF16, 3, k ** -0.5).cuda()
    fx, fdy, out = far(x), far(dy), far(dy)
    y, pre = T.linear(x, w, residual=dy, act="silu", pre=True)
    T.linear(fx, w, residual=fdy, act="silu", out=out)
    assert torch.equal(out, y)
    fpre = out.copy_(pre)
    for got, want in zip(T.linear_grad(fdy, fx, w, fpre, act="silu"), T.linear_grad(dy, x, w, pre, act="silu")):
        assert torch.equal(got, want)
    norms = dict(post=dict(kind="rms"), pre=dict(kind="layer"))
    r, h, st = T.residual_norm(dy, pre, stats=True, **norms)
    fr, fh, fst = T.residual_norm(fdy, fpre, stats=True, **norms)
    assert torch.equal(fr, r) and torch.equal(fh, h) and torch.equal(fst, st)
    for got, want in zip(T.residual_norm_grad(fdy, fpre, fdy, fpre, st, **norms),
                         T.residual_norm_grad(dy, pre, dy, pre, st, **norms)):
        assert got is None and want is None or torch.equal(got, want)
    labels = (torch.arange(m, dtype=torch.int32) % n).cuda()
    q, fq = T.label_log_probs(dy, labels, top=3, entropy=True), T.label_log_probs(fdy, labels, top=3, entropy=True)
    for a, b in zip(q, fq):
        assert torch.equal(a, b)
    g = normal((m,), F32, 9).cuda()
    assert torch.equal(T.label_log_probs_grad(fdy, labels, q.stats, g), T.label_log_probs_grad(dy, labels, q.stats, g))


def test_logits_past_32_bits():
    """One array of 2.2e9 logits: the last rows as by themselves."""
    note("logits past 32 bits")
    m, c = 43_000, 51_201
    x = torch.zeros(m, c, dtype=BF16, device="cuda")
    tail = normal((3, c), BF16, 1).cuda()
    x[m - 3:] = tail
    labels = torch.full((m,), 17, dtype=torch.int32, device="cuda")
    r = T.label_log_probs(x, labels, top=2, entropy=True)
    for a, b in zip(r, T.label_log_probs(x[m - 2000:].contiguous(), labels[:2000], top=2, entropy=True)):
        close(a[m - 3:], b[-3:].double().cpu(), 1e-5, F32)
    assert (r.top_ids[m - 5].cpu() == torch.tensor([0, 1])).all()
    dx = T.label_log_probs_grad(x, labels, r.stats, torch.ones(m, device="cuda"), out=torch.empty_like(x))
    want = T.label_log_probs_grad(tail, labels[:3], r.stats[m - 3:].contiguous(), torch.ones(3, device="cuda"))
    assert torch.equal(dx[m - 3:], want)


def test_wrapper_refusals():
    note("refusals")
    x = torch.zeros(8, 16, device="cuda")
    w, v = torch.zeros(16, 16, device="cuda"), torch.zeros(16, device="cuda")
    off = torch.tensor([0, 8], device="cuda")
    ids = torch.zeros(8, dtype=torch.int32, device="cuda")
    s2, s4, one = torch.zeros(8, 2, device="cuda"), torch.zeros(8, 4, device="cuda"), torch.zeros(8, device="cuda")
    rms = dict(kind="rms")
    bad = [
        lambda: T.linear(x, w.t()), lambda: T.linear(x, w.to(BF16)), lambda: T.linear(x, w[:8]), lambda: T.linear(x, w, v[:8]),
        lambda: T.linear(x, w, v.to(BF16)), lambda: T.linear(x, w, residual=x[:4]), lambda: T.linear(x, w, residual=x.to(BF16)),
        lambda: T.linear(x, w, out=x), lambda: T.linear(x, w, residual=x, out=x), lambda: T.linear(x, w, act="tanh"),
        lambda: T.linear(x[0], w), lambda: T.linear(x.double(), w), lambda: T.linear(x, w.cpu()), lambda: T.linear(x, v),
        lambda: T.linear(x, w, out=torch.empty(8, 16, device="cuda"), out_dtype=BF16), lambda: T.linear(x.t(), w[:8]),
        lambda: T.linear_grad(x, x, w, act="silu"), lambda: T.linear_grad(x.to(BF16), x, w), lambda: T.linear_grad(x[:, :8], x, w),
        lambda: T.linear_grad(x, x, w, x[:4], act="silu"), lambda: T.linear_grad(x, x, w, weight_dtype=torch.float64),
        lambda: T.residual_norm(x, x.double()), lambda: T.residual_norm(x[:4], x), lambda: T.residual_norm(x, x, gate=v[:8]),
        lambda: T.residual_norm(x, x, gate=v, off=off), lambda: T.residual_norm(x, x, off=off.int()),
        lambda: T.residual_norm(x, x, post=dict(kind="batch")), lambda: T.residual_norm(x, x, pre=dict(weight=v[:3])),
        lambda: T.residual_norm(x, x, pre=dict(gamma=v)), lambda: T.residual_norm(x, x, out=x),
        lambda: T.residual_norm(x, x, out_h=torch.empty_like(x)), lambda: T.residual_norm(x, x.cpu()),
        lambda: T.residual_norm_grad(x, x, x, x, s4), lambda: T.residual_norm_grad(x, None, x, x, s4, pre=rms),
        lambda: T.residual_norm_grad(x, x, x, x, None, pre=rms), lambda: T.residual_norm_grad(x, x, x, x, s4[:4], pre=rms),
        lambda: T.residual_norm_grad(x.to(BF16), x, x, x, s4, pre=rms), lambda: T.residual_norm_grad(x, x.to(BF16), x, x, s4, pre=rms),
        lambda: T.label_log_probs(x, ids.long()), lambda: T.label_log_probs(x, ids[:4]), lambda: T.label_log_probs(x, ids.cpu()),
        lambda: T.label_log_probs(x.double(), ids), lambda: T.label_log_probs(x[0], ids),
        lambda: T.label_log_probs_grad(x, ids, s2, one.double()), lambda: T.label_log_probs_grad(x, ids, s2[:4], one),
        lambda: T.label_log_probs_grad(x, ids, s2, one, out=x), lambda: T.label_log_probs_grad(x, ids, s2.t(), one),
        lambda: T.label_log_probs_grad(x, ids, s2, one, out=torch.empty(8, 15, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted", i)
    for call in (lambda: T.residual_norm(x.to(F16), x.to(BF16)), lambda: T.residual_norm(x, x, post=dict(eps=-1.0)),
                 lambda: T.residual_norm(*[torch.zeros(2, 8193, device="cuda")] * 2), lambda: T.label_log_probs(x, ids, top=17),
                 lambda: T.label_log_probs(x, ids, 0.0), lambda: T.label_log_probs(x, ids, top=-1)):
        with pytest.raises(T.TaurusError):
            call()
    wide = torch.zeros(8, 32, device="cuda")  # columns of one wide array do not overlap
    T.linear(wide[:, :16], w, out=wide[:, 16:])
    T.residual_norm(wide[:, :16], wide[:, :16], out=wide[:, 16:])


def test_broken_offsets_touch_nothing_else():
    """Offsets outside [0, m] are clamped: rows around the arrays stay."""
    note("offsets outside the rows")
    for dtype in (F32, BF16):
        big, big_h = (torch.full((300, 16), 2.0, dtype=dtype, device="cuda") for _ in range(2))
        x = torch.ones(100, 16, dtype=dtype, device="cuda")
        gate = torch.ones(3, 16, device="cuda")
        for off in ([-50, 40, 10_000, 2 ** 40], [60, 20, 90, 5], [100, 0, 100, 0]):
            off = torch.tensor(off, device="cuda")
            y, h, st = T.residual_norm(x, x, gate=gate, off=off, pre=dict(kind="rms"), out=big[100:200], out_h=big_h[100:200], stats=True)
            T.residual_norm_grad(x, x, y, x, torch.ones_like(st), gate=gate, off=off, pre=dict(kind="rms"))
            for t in (big, big_h):
                assert (t[:100] == 2).all() and (t[200:] == 2).all()
    off = torch.tensor([-50, 40, 10_000, 2 ** 40], device="cuda")
    assert (T.residual_norm(x, x, gate=gate, off=off)[0] == 2).all()


def test_blocks_and_a_head_in_a_model():
    """Two residual blocks around GraphSAGE layers and a two-map classifier,
    against the same model in 64 bits."""
    from fixtures import workloads as WL
    from tests import harness as H
    note("blocks and a head in a model")
    n, d, c = WL.SAGE_RMAT_4K.n, 32, 47
    src, dst = WL.graph(WL.SAGE_RMAT_4K)
    row_off, col_dst = T.build_csr(n, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda())
    x = normal((n + 5, d), F32, 1)  # rows behind the vertices stay out
    gate, w2, b2 = normal((d,), F32, 2), normal((d,), F32, 3), normal((d,), F32, 4)
    gates, off = normal((3, d), F32, 5), ranges([n // 2, 0, n - n // 2])
    wc = [normal((d, 2 * d), F32, 6 + i, 0.2).numpy() for i in range(2)]
    lw, lb, cw, cb = normal((d, 40), F32, 8, 0.2), normal((40,), F32, 9), normal((40, c), F32, 10, 0.3), normal((c,), F32, 11)
    labels = torch.randint(-1, c, (n,), generator=torch.Generator().manual_seed(12), dtype=torch.int32)
    layers = [dict(agg=N.SAGE_MEAN, d_in=d, d_out=d, weight_cat=wc[0], bias=None, relu=True, layer=1,
                   residual=dict(scale=0.5, gate=gate.cuda(), pre=dict(kind="layer", weight=w2.cuda(), bias=b2.cuda()))),
              dict(agg=N.SAGE_MEAN, d_in=d, d_out=d, weight_cat=wc[1], bias=None, relu=False, layer=2,
                   residual=dict(gate=gates.cuda(), off=off.cuda(), post=dict(kind="rms"), pre=dict(kind="rms")))]
    head = dict(linear=[dict(weight=lw.cuda(), bias=lb.cuda(), act="gelu"), dict(weight=cw.cuda(), bias=cb.cuda())],
                labels=labels.cuda(), top=3, entropy=True, scale=0.7)
    outs, stats = T.run_layers(n, row_off, col_dst, x.cuda()[:n], layers, chunk=1024, head=head)
    assert len(outs) == 3 and len(stats) == 2

    def sage(h, w, relu):
        W = torch.from_numpy(w).double()
        s = torch.zeros(n, d, dtype=torch.float64)
        s.index_add_(0, torch.from_numpy(dst).long(), h[torch.from_numpy(src).long()])
        deg = torch.bincount(torch.from_numpy(dst).long(), minlength=n).clamp(min=1).double().unsqueeze(1)
        z = (s / deg) @ W[:, :d] + h @ W[:, d:]
        return z.clamp(min=0) if relu else z

    def norm(v, kind, w=None, b=None):
        zero = torch.zeros(v.shape).double()
        return norm_of(v, zero, dict(kind=kind, weight=w, bias=b), d)[0]
    h = x[:n].double()
    y1 = h + 0.5 * gate.double() * sage(h, wc[0], True)
    h = norm(y1, "layer", w2, b2)
    y2 = y1 + gate_rows(gates, off.tolist(), n, d)[0] * norm(sage(h, wc[1], False), "rms")
    h = norm(y2, "rms")
    for got, ref in zip(outs, (y1, y2)):
        r = H.compare(got.cpu().numpy(), ref.numpy(), H.RTOL[N.F32])
        assert r["n_bad"] == 0, r
    z = h @ lw.double() + lb.double()
    logits = (z * phi_cdf(z)) @ cw.double() + cb.double()
    lp = torch.log_softmax(0.7 * logits, 1)
    a = outs[2]
    known = labels >= 0
    want = torch.where(known, lp.gather(1, labels.clamp(min=0).long().unsqueeze(1)).squeeze(1), 0.0)
    for got, ref in ((a.logp, want), (a.entropy, -(lp * lp.exp()).sum(1)), (a.top_logp, lp.topk(3).values)):
        r = H.compare(got.cpu().view(n, -1).numpy(), ref.view(n, -1).numpy(), H.RTOL[N.F32])
        assert r["n_bad"] == 0, r
    assert (lp.gather(1, a.top_ids.cpu().long()) - lp.topk(3).values).abs().max() < 1e-4
    # on another stream, into given outputs, from a padded input
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    given = [torch.empty_like(o) for o in outs[:2]]
    again, _ = T.run_layers(n, row_off, col_dst, x.cuda(), layers, chunk=1024, head=head, outs=given, stream=s)
    for p, q in zip([*again[:2], *again[2]], [*outs[:2], *outs[2]]):
        assert torch.equal(p, q)
    assert again[0] is given[0] and again[1] is given[1]


def test_blocks_behind_a_layer_that_streams_from_the_host():
    """x in pinned host memory through a plain layer, then a block and a head on
    the device; a block on the host's rows is refused before anything is
    written."""
    from fixtures import workloads as WL
    from tests import harness as H
    note("blocks behind a streamed layer")
    n, d = WL.SAGE_RMAT_4K.n, 32
    src, dst = WL.graph(WL.SAGE_RMAT_4K)
    row_off, col_dst = T.build_csr(n, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda())
    x = normal((n, d), F32, 1)
    host = x.pin_memory()
    layers = [dict(agg=N.SAGE_MEAN, d_in=d, d_out=d, weight_cat=normal((d, 2 * d), F32, 2 + i, 0.2).numpy(), bias=None,
                   relu=True, layer=1 + i) for i in range(2)]
    layers[1]["residual"] = dict(gate=normal((d,), F32, 4).cuda(), pre=dict(kind="rms"))
    want, _ = T.run_layers(n, row_off, col_dst, x.cuda(), layers, chunk=1024, head=dict(top=3, entropy=True))
    first = torch.empty(n, d, device="cuda")
    got, _ = T.run_layers(n, row_off, col_dst, host, layers, chunk=1024, outs=[first, None], head=dict(top=3, entropy=True))
    assert got[0] is first and got[1].is_cuda
    for a, b in ((got[0], want[0]), (got[1], want[1]), (got[2].entropy, want[2].entropy), (got[2].top_logp, want[2].top_logp)):
        r = H.compare(a.view(n, -1).cpu().numpy(), b.view(n, -1).double().cpu().numpy(), H.RTOL[N.F32])
        assert r["n_bad"] == 0, r
    first.fill_(7.0)
    for rows, outs in ((host, [None, None]), (x.cuda(), [first, host])):
        with pytest.raises(ValueError, match="where the graph is"):
            T.run_layers(n, row_off, col_dst, rows, [layers[1], layers[1]], chunk=1024, outs=outs)
    assert (first == 7.0).all()
