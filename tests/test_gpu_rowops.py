"""Row lookup, grouped linear maps, group norm and their gradients against
plain 64-bit implementations (needs an MI355X).

Tolerances follow from the arithmetic: u = 2^-24 is half a step of fp32, a sum
of n terms in any order is off by at most n u times the sum of their sizes
(matrix cores: twice that, their adder may truncate), and the stored result
by half a step of its type.
"""
import sys

import pytest
import torch

import paper_2607_17374_amd as T
from paper_2607_17374_amd import _native as N

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}        # eps / 2
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}     # least positive value (fp16: half of it)


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def note(msg):
    print(f"[case] {msg}", flush=True)
    sys.stdout.flush()


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def strided(t, pad, lead=0):
    """A device copy of t whose rows lie pad + lead values apart from dense,
    lead of them in front; what surrounds it is NaN."""
    m, d = t.shape
    wide = torch.full((m, lead + d + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, lead:lead + d] = t.cuda()
    return wide[:, lead:lead + d]


def close(got, ref, tol, dtype, what=""):
    """|got - ref| <= tol + half a step of dtype, everywhere."""
    got = got.double().cpu()
    bound = tol + HALF[dtype] * (ref.abs() + tol) + TINY[dtype]
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / bound)[bad].max()),
                           bad.nonzero()[:4].tolist())


# ----------------------------------------------------------------- lookup --

@pytest.mark.parametrize("din", DTYPES)
@pytest.mark.parametrize("dout", DTYPES)
@pytest.mark.parametrize("n,m,d", [(1, 1, 1), (7, 5, 3), (100, 64, 8), (50, 1000, 47), (1000, 333, 128), (64, 9, 172),
                                   (33, 70, 257), (5, 3, 2056), (10, 0, 16), (0, 4, 12)])
def test_lookup(din, dout, n, m, d):
    note(f"lookup {din} -> {dout} n={n} m={m} d={d}")
    g = torch.Generator().manual_seed(n * 1000 + m)
    table = normal((n, d), din, 3 * n + d)
    ids = torch.randint(0, max(n, 1), (m,), generator=g, dtype=torch.int32)
    if m > 2:
        ids[0], ids[1], ids[m // 2] = -1, n, -2 ** 31
    scale = 1.7
    out = T.lookup_rows(table.cuda(), ids.cuda(), scale, out_dtype=dout)
    assert out.dtype == dout and tuple(out.shape) == (m, d)
    known = (ids >= 0) & (ids < n)
    ref = torch.zeros(m, d, dtype=torch.float64)
    # the scale is an fp32 value to the library
    s32 = float(torch.tensor(scale, dtype=F32))
    ref[known] = table.double()[ids[known].long()] * s32
    close(out, ref, 2 * U * ref.abs(), dout, "lookup")
    assert (out.cpu()[~known] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,pad,lead", [(16, 8, 0), (16, 3, 0), (16, 0, 1), (12, 4, 4), (5, 1, 2), (64, 64, 8)])
def test_lookup_strided(dtype, d, pad, lead):
    note(f"lookup strided {dtype} d={d} pad={pad} lead={lead}")
    table = strided(normal((40, d), dtype, 1), pad, lead)
    ids = torch.tensor([3, 39, -1, 0, 3, 17, 40, 8], dtype=torch.int32).cuda()
    wide = torch.full((8, lead + d + pad), 7.0, dtype=dtype, device="cuda")
    out = wide[:, lead:lead + d]
    assert T.lookup_rows(table, ids, out=out) is out
    ref = torch.zeros(8, d, dtype=dtype, device="cuda")
    ref[[0, 1, 3, 4, 5, 7]] = table[[3, 39, 0, 3, 17, 8]]
    assert torch.equal(out, ref)  # a scale of one changes no bit
    around = torch.cat([wide[:, :lead], wide[:, lead + d:]], 1)
    assert (around == 7.0).all()


def test_lookup_special_rows():
    """Rows of infinities and NaN reach only those that ask for them."""
    note("lookup special rows")
    t = torch.ones(4, 8, device="cuda")
    t[1], t[2] = float("inf"), float("nan")
    out = T.lookup_rows(t, torch.tensor([0, -1, 1, 2, 3, 99], dtype=torch.int32).cuda(), 0.5).cpu()
    assert (out[0] == 0.5).all() and (out[1] == 0).all() and torch.isinf(out[2]).all()
    assert torch.isnan(out[3]).all() and (out[4] == 0.5).all() and (out[5] == 0).all()


def test_lookup_far_rows():
    """Rows whose offsets pass 32 bits (2.6e9 values)."""
    note("lookup far rows")
    n, d = 20_000_003, 128
    table = torch.empty(n, d, dtype=BF16, device="cuda")
    ids = torch.tensor([n - 1, 0, 16_777_217, n - 2], dtype=torch.int32).cuda()
    rows = normal((4, d), BF16, 5).cuda()
    table[ids.long()] = rows
    assert torch.equal(T.lookup_rows(table, ids), rows)
    grad = T.lookup_rows_grad(rows, ids, n, out=table)
    assert torch.equal(grad[ids.long()], rows)
    assert not grad[1:1000].any() and not grad[n - 1000:n - 2].any() and not grad[16_777_218:16_778_000].any()


def grad_reference(grad, ids, n, scale):
    """Sums, and sums of sizes and counts per row for the tolerance."""
    keep = (ids >= 0) & (ids < n)
    at = ids[keep].long()
    total = torch.zeros(n, grad.shape[1], dtype=torch.float64)
    size = torch.zeros_like(total)
    total.index_add_(0, at, grad.double()[keep])
    size.index_add_(0, at, grad.double()[keep].abs())
    count = torch.bincount(at, minlength=n).double().unsqueeze(1)
    return total * scale, size * abs(scale), count


def make_ids(kind, m, n, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        ids = torch.randint(0, n, (m,), generator=g)
    elif kind == "one":
        ids = torch.full((m,), n - 1)
    elif kind == "hubs":
        ids = torch.where(torch.rand(m, generator=g) < 0.7, torch.randint(0, 3, (m,), generator=g) * (n // 3),
                          torch.randint(0, n, (m,), generator=g))
    elif kind == "runs":  # each id a run of 31 to 65 places: they end inside and at tiles
        ids = torch.repeat_interleave(torch.arange(n), 31 + torch.arange(n) % 35)[:m]
        ids = torch.cat([ids, torch.zeros(m - ids.numel(), dtype=torch.int64)])
    else:  # none
        ids = torch.full((m,), -1)
    ids = ids.to(torch.int32)
    if kind == "uniform" and m > 4:
        ids[1], ids[m // 2], ids[m - 1] = -1, n, 2 ** 31 - 1
    return ids


@pytest.mark.parametrize("m", [0, 1, 2, 63, 65, 1000, 1024, 1025, 4096, 4097, 40_000, 65_536,
                               65_537, 300_000])
@pytest.mark.parametrize("kind", ["uniform", "one", "hubs", "runs", "none"])
def test_lookup_grad(m, kind):
    n, d, scale = 257, 40, -0.75
    note(f"lookup_grad {kind} m={m}")
    ids = make_ids(kind, m, n, m)
    grad = normal((m, d), F32, m + 1)
    out = T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, scale)
    ref, size, count = grad_reference(grad, ids, n, scale)
    close(out, ref, (count + 2) * U * size, F32, kind)
    assert (out.cpu()[count[:, 0] == 0] == 0).all()
    again = T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, scale)
    assert torch.equal(out, again)  # no order is left to chance


@pytest.mark.parametrize("n", [1, 511, 512, 70_001, 1_000_003])
@pytest.mark.parametrize("m", [100, 1500, 5000, 70_000])
def test_lookup_grad_tables(n, m):
    """Tables of one row to many more than there are ids (most rows then are
    filled with zeros beforehand), ids of one to three sort digits."""
    note(f"lookup_grad table n={n} m={m}")
    ids = make_ids("uniform", m, n, n + m)
    grad = normal((m, 12), F32, n)
    out = torch.full((n, 12), 5.0, device="cuda")
    T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, out=out)
    ref, size, count = grad_reference(grad, ids, n, 1.0)
    close(out, ref, (count + 2) * U * size, F32, "tables")


@pytest.mark.parametrize("din", DTYPES)
@pytest.mark.parametrize("dout", DTYPES)
@pytest.mark.parametrize("d", [1, 3, 8, 44, 128, 257, 600])
@pytest.mark.parametrize("m", [90, 3000])
def test_lookup_grad_types(din, dout, d, m):
    note(f"lookup_grad {din} -> {dout} d={d} m={m}")
    n = 61
    ids = make_ids("hubs", m, n, d)
    grad = normal((m, d), din, d + 1)
    g = strided(grad, 5, 3) if d % 2 else grad.cuda()
    out = T.lookup_rows_grad(g, ids.cuda(), n, 0.5, out_dtype=dout)
    ref, size, count = grad_reference(grad, ids, n, 0.5)
    close(out, ref, (count + 2) * U * size, dout, "types")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [0, 5, 900, 5000])
def test_lookup_grad_accumulates(dtype, m):
    """Named rows get the sum added with one rounding; others, NaN among them,
    are not touched; padding columns neither."""
    note(f"lookup_grad accumulate {dtype} m={m}")
    n, d = 3001, 24
    ids = make_ids("uniform", m, n, 7)
    ids[ids == 5] = 6
    grad = normal((m, d), dtype, 8)
    old = normal((n, d), dtype, 9)
    old[5] = float("nan")
    wide = torch.full((n, d + 8), 3.0, dtype=dtype, device="cuda")
    wide[:, :d] = old.cuda()
    out = T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, 2.0, out=wide[:, :d], accumulate=True)
    ref, size, count = grad_reference(grad, ids, n, 2.0)
    named = count[:, 0] > 0
    total = ref + old.double()
    close(out[named.cuda()], total[named], ((count + 2) * U * size + U * total.abs())[named], dtype, "accumulate")
    rest = out.cpu()[~named]
    assert torch.equal(rest.view(torch.int32 if dtype == F32 else torch.int16),
                       old[~named].contiguous().view(torch.int32 if dtype == F32 else torch.int16))
    assert (wide[:, d:] == 3.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [3, 7, 12, 20, 257])
@pytest.mark.parametrize("m", [60, 3000])
def test_lookup_grad_accumulates_to_any_width(dtype, d, m):
    """A row's last vector covers values of the one before it: each value is
    added to once."""
    note(f"lookup_grad accumulate {dtype} d={d} m={m}")
    n = 41
    ids = make_ids("uniform", m, n, d)
    grad, old = normal((m, d), dtype, 8), normal((n, d), dtype, 9)
    out = strided(old, 3, 1)
    T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, 2.0, out=out, accumulate=True)
    ref, size, count = grad_reference(grad, ids, n, 2.0)
    total = ref + old.double()
    close(out, total, (count + 2) * U * size + U * total.abs(), dtype, "accumulate")


@pytest.mark.parametrize("n,d", [(70_001, 2), (3_000_017, 1)])
def test_lookup_grad_of_millions(n, d):
    """Over 4,194,304 ids: the sort's tiles are grouped."""
    m = 4_300_003
    note(f"lookup_grad of millions m={m} n={n} d={d}")
    ids = make_ids("uniform", m, n, 1)
    ids[:1_000_000] = n // 2  # one id of many tiles
    grad = normal((m, d), F32, 2)
    out = T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, 0.5)
    ref, size, count = grad_reference(grad, ids, n, 0.5)
    close(out, ref, (count + 2) * U * size, F32, "millions")
    assert torch.equal(out, T.lookup_rows_grad(grad.cuda(), ids.cuda(), n, 0.5))


def test_lookup_grad_special_values():
    """An id's infinities and NaN stay in its own row, those of padded places
    reach none."""
    note("lookup_grad special values")
    for m in (200, 2000):
        grad = torch.ones(m, 8)
        ids = (torch.arange(m) % 50).to(torch.int32)
        ids[ids == 49] = -1
        grad[ids == -1] = float("nan")
        grad[3], grad[7] = float("inf"), float("nan")
        out = T.lookup_rows_grad(grad.cuda(), ids.cuda(), 60).cpu()
        assert torch.isinf(out[3]).all() and torch.isnan(out[7]).all()
        rest = [i for i in range(60) if i not in (3, 7)]
        assert torch.isfinite(out[rest]).all() and (out[49:] == 0).all()


# ---------------------------------------------------------- grouped linear --

def ranges(sizes, lead=0):
    off = [lead]
    for s in sizes:
        off.append(off[-1] + s)
    return torch.tensor(off, dtype=torch.int64)


LINEAR = [  # type sizes, d_in, d_out
    ([1], 1, 1), ([0, 3, 0], 5, 7), ([1, 1, 1, 1], 16, 4), ([130, 0, 127, 128, 129], 64, 64), ([300], 100, 47),
    ([5, 200, 61], 128, 256), ([77], 33, 130), ([256, 1], 1024, 40), ([40, 40], 200, 129), ([0, 0], 8, 8),
    ([3] * 150, 24, 20), ([513], 8, 300), ([130, 70], 14, 280), ([90], 15, 9), ([64, 5], 22, 31), ([129], 71, 133),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LINEAR)))
def test_grouped_linear(dtype, case):
    sizes, k, n = LINEAR[case]
    note(f"grouped_linear {dtype} {sizes[:6]} {k} -> {n}")
    off = ranges(sizes)
    m, g = int(off[-1]), len(sizes)
    x, w = normal((m, k), dtype, case), normal((g, k, n), dtype, case + 1, k ** -0.5)
    bias = normal((g, n), F32, case + 2)
    out_dtype = [dtype, F32, BF16][case % 3]
    out = T.grouped_linear(x.cuda(), off.cuda(), w.cuda(), bias.cuda(), out_dtype=out_dtype)
    plain = T.grouped_linear(x.cuda(), off.cuda(), w.cuda(), out_dtype=F32)
    ref, size = torch.zeros(m, n, dtype=torch.float64), torch.zeros(m, n, dtype=torch.float64)
    for i in range(g):
        r = slice(int(off[i]), int(off[i + 1]))
        ref[r] = x[r].double() @ w[i].double()
        size[r] = x[r].double().abs() @ w[i].double().abs()
    close(plain, ref, 2 * (k + 1) * U * size, F32, "no bias")
    at = torch.repeat_interleave(torch.arange(g), torch.tensor(sizes))
    close(out, ref + bias.double()[at], 2 * (k + 2) * U * (size + bias.double().abs()[at]), out_dtype, "bias")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k,n,pad,lead", [(64, 64, 8, 8), (64, 64, 3, 1), (40, 72, 0, 1), (17, 9, 2, 0), (128, 260, 4, 4)])
def test_grouped_linear_strided_and_outside(dtype, k, n, pad, lead):
    """Rows before the first and behind the last type stay as they were, rows
    of NaN outside and in other types reach no one."""
    note(f"grouped_linear strided {dtype} {k} -> {n} pad={pad} lead={lead}")
    off = ranges([70, 0, 33, 140], lead=9)
    m = int(off[-1]) + 11
    x = normal((m, k), dtype, 1)
    x[:9] = float("nan")
    x[int(off[-1]):] = float("nan")
    x[int(off[2]):int(off[3])] = float("inf")  # the third type
    w = normal((4, k, n), dtype, 2, k ** -0.5)
    wide = torch.full((m, lead + n + pad), 5.0, dtype=dtype, device="cuda")
    out = wide[:, lead:lead + n]
    T.grouped_linear(strided(x, pad, lead), off.cuda(), w.cuda(), out=out)
    got = out.cpu()
    assert (got[:9] == 5.0).all() and (got[int(off[-1]):] == 5.0).all()
    assert not torch.isfinite(got[int(off[2]):int(off[3])]).any()
    for i in (0, 3):
        r = slice(int(off[i]), int(off[i + 1]))
        ref = x[r].double() @ w[i].double()
        close(got[r], ref, 2 * (k + 1) * U * (x[r].double().abs() @ w[i].double().abs()), dtype, i)
    assert (torch.cat([wide[:, :lead], wide[:, lead + n:]], 1) == 5.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LINEAR)))
def test_grouped_linear_grad(dtype, case):
    sizes, k, n = LINEAR[case]
    note(f"grouped_linear_grad {dtype} {sizes[:6]} {k} -> {n}")
    off = ranges(sizes)
    m, g = int(off[-1]), len(sizes)
    x, w = normal((m, k), dtype, case), normal((g, k, n), dtype, case + 1, k ** -0.5)
    dy = normal((m, n), dtype, case + 2)
    wd = [F32, dtype][case % 2]
    dx, dw, db = T.grouped_linear_grad(dy.cuda(), x.cuda(), off.cuda(), w.cuda(), weight_dtype=wd)
    assert dx.dtype == dtype and dw.dtype == wd and db.dtype == F32
    for i in range(g):
        r = slice(int(off[i]), int(off[i + 1]))
        rows = sizes[i]
        xd, yd, wdbl = x[r].double(), dy[r].double(), w[i].double()
        close(dx[r], yd @ wdbl.T, 2 * (n + 1) * U * (yd.abs() @ wdbl.abs().T), dtype, ("dx", i))
        close(dw[i], xd.T @ yd, 2 * (rows + 1) * U * (xd.abs().T @ yd.abs()), wd, ("dw", i))
        close(db[i], yd.sum(0), 2 * (rows + 1) * U * yd.abs().sum(0), F32, ("db", i))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sizes,k,n", [([2000, 1, 0, 257, 256, 3100], 24, 40), ([700] * 9, 130, 20), ([5000], 64, 136),
                                       ([1] * 700 + [900], 12, 12)])
def test_grouped_linear_grad_long_types(dtype, sizes, k, n):
    """Types of many units: their sums are joined from the workspace; rows
    outside, of NaN, reach no gradient; equal calls give equal bits."""
    off = ranges(sizes, lead=3)
    m, g = int(off[-1]) + 5, len(sizes)
    note(f"grouped_linear_grad long {dtype} m={m} {k} -> {n}")
    x, dy = normal((m, k), dtype, 1), normal((m, n), dtype, 2)
    for t in (x, dy):
        t[:3], t[m - 5:] = float("nan"), float("nan")
    w = normal((g, k, n), dtype, 3, k ** -0.5)
    xs, ys = strided(x, 8, 8), strided(dy, 3, 1)
    _, dw, db = T.grouped_linear_grad(ys, xs, off.cuda(), w.cuda(), need=("weight", "bias"))
    for i in range(g):
        r = slice(int(off[i]), int(off[i + 1]))
        xd, yd = x[r].double(), dy[r].double()
        close(dw[i], xd.T @ yd, 2 * (sizes[i] + 1) * U * (xd.abs().T @ yd.abs()), F32, ("dw", i))
        close(db[i], yd.sum(0), 2 * (sizes[i] + 1) * U * yd.abs().sum(0), F32, ("db", i))
    none, dw2, none2 = T.grouped_linear_grad(ys, xs, off.cuda(), w.cuda(), need=("weight",))
    assert none is None and none2 is None and torch.equal(dw, dw2)
    none, none2, db2 = T.grouped_linear_grad(ys, xs, off.cuda(), w.cuda(), need=("bias",))
    assert none is None and none2 is None and torch.equal(db, db2)


WEIGHT = [  # type sizes, d_in, d_out
    ([9_000, 0, 17_000, 1] + [40, 0, 333, 65] * 14, 1024, 320),  # more tiles than workgroups, long types among short
    ([299_223, 0, 777], 24, 40),                                 # units of more than 256 rows
    ([40_000], 2048, 2048),                                      # units of more than 8,192 rows
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(WEIGHT)))
def test_grouped_linear_grad_many_units(dtype, case):
    """Workgroups that take several tiles of several units."""
    sizes, k, n = WEIGHT[case]
    off, g = ranges(sizes), len(sizes)
    m = int(off[-1])
    note(f"grouped_linear_grad many units {dtype} m={m} types={g} {k} -> {n}")
    x, dy = normal((m, k), dtype, 1).cuda(), normal((m, n), dtype, 2).cuda()
    w = torch.zeros(g, k, n, dtype=dtype, device="cuda")
    wd = [dtype, F32][case % 2]
    _, dw, db = T.grouped_linear_grad(dy, x, off.cuda(), w, need=("weight", "bias"), weight_dtype=wd)
    for i in range(g):
        r = slice(int(off[i]), int(off[i + 1]))
        xd, yd = x[r].double(), dy[r].double()
        xt = xd.t().contiguous()
        tol = 2 * (sizes[i] + 1) * U
        for got, ref, size, out in ((dw[i], xt @ yd, xt.abs() @ yd.abs(), wd), (db[i], yd.sum(0), yd.abs().sum(0), F32)):
            bound = tol * size + HALF[out] * (ref.abs() + tol * size) + TINY[out]
            assert ((got.double() - ref).abs() <= bound).all(), (i, sizes[i])
    _, dw2, _ = T.grouped_linear_grad(dy, x, off.cuda(), w, need=("weight",), weight_dtype=wd)
    _, _, db2 = T.grouped_linear_grad(dy, x, off.cuda(), w, need=("bias",))
    assert torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,n", [(14_000, 72, 300), (66_100, 40, 24), (14_000, 33, 301), (66_100, 301, 17),
                                   (40_000, 129, 128)])
def test_grouped_linear_many_tiles(dtype, m, k, n):
    """More tiles than are resident at once: workgroups take several."""
    note(f"grouped_linear many tiles {dtype} {m} rows {k} -> {n}")
    off = ranges([m // 3, 0, 1, m // 5 + 7, m - m // 3 - m // 5 - 8])
    x, dy = normal((m, k), dtype, 1), normal((m, n), dtype, 2)
    w, b = normal((5, k, n), dtype, 3, k ** -0.5), normal((5, n), F32, 4)
    y = T.grouped_linear(x.cuda(), off.cuda(), w.cuda(), b.cuda()).cpu()
    dx = T.grouped_linear_grad(dy.cuda(), x.cuda(), off.cuda(), w.cuda(), need=("x",))[0].cpu()
    for g in range(5):
        r = slice(int(off[g]), int(off[g + 1]))
        wg, bg = w[g].double(), b[g].double()
        size = x[r].double().abs() @ wg.abs() + bg.abs()
        close(y[r], x[r].double() @ wg + bg, 2 * (k + 1) * U * size, dtype, (g, "y"))
        size = dy[r].double().abs() @ wg.abs().T
        close(dx[r], dy[r].double() @ wg.T, 2 * (n + 1) * U * size, dtype, (g, "dx"))


def test_grouped_linear_differences():
    """dx, dW, db against differences of the 64-bit map along random
    directions: the map is bilinear, so central differences are exact."""
    note("grouped_linear differences")
    off = ranges([37, 90, 0, 13])
    m, g, k, n = 140, 4, 20, 28
    x, w, b = normal((m, k), F32, 1), normal((g, k, n), F32, 2), normal((g, n), F32, 3)
    c = normal((m, n), F32, 4)
    at = torch.repeat_interleave(torch.arange(g), off[1:] - off[:-1])

    def loss(x, w, b):
        return ((torch.einsum("mk,mkn->mn", x, w[at]) + b[at]) * c.double()).sum()
    dx, dw, db = T.grouped_linear_grad(c.cuda(), x.cuda(), off.cuda(), w.cuda())
    X, W, B = x.double(), w.double(), b.double()
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        v = normal(tuple(grad.shape), F32, 10 + which).double()
        h = 0.5
        hi, lo = [X, W, B], [X, W, B]
        hi[which], lo[which] = hi[which] + h * v, lo[which] - h * v
        diff = float((loss(*hi) - loss(*lo)) / (2 * h))
        got = float((grad.double().cpu() * v).sum())
        size = float((grad.double().cpu().abs() * v.abs()).sum())
        assert abs(got - diff) <= 2 * (m + 2) * U * 40 * size + 1e-9


# -------------------------------------------------------------- group norm --
# D bounds the number of additions any value passes on its way into a mean:
# 16 values a lane, 8 joins of lanes or waves, at most 1024 / 4 merges of a
# unit's rows (two roundings each), 12 halvings, then a workgroup's sum over
# units.
D = 16 + 8 + 512 + 24 + 40


def norm_reference(x, groups, w, b, off, eps, act):
    """(y, mean, rstd, tolerances) of the definition in 64 bits."""
    m, d = x.shape
    cg = d // groups
    X = x.double().view(m, groups, cg)
    W = torch.ones(d).double() if w is None else w.double()
    B = torch.zeros(d).double() if b is None else b.double()
    segs = [(r, r + 1) for r in range(m)] if off is None else [(int(p), int(q)) for p, q in zip(off[:-1], off[1:])]
    mean = torch.zeros(len(segs), groups, dtype=torch.float64)
    rstd, tmean, trel = torch.zeros_like(mean), torch.zeros_like(mean), torch.zeros_like(mean)
    y = torch.full((m, d), float("nan"), dtype=torch.float64)
    z, tz = y.clone(), y.clone()
    for s, (p, q) in enumerate(segs):
        if p == q:
            continue
        v = X[p:q]
        mu = v.mean((0, 2))
        var = ((v - mu.view(1, -1, 1)) ** 2).mean((0, 2))
        r = (var + eps) ** -0.5
        top = v.abs().amax((0, 2))
        # deviations are off by the mean's error; its square enters the variance
        em = D * U * top
        ev = (2 * D * U * var + 2 * em * em + 2 * em * var.sqrt() * U * D + 4 * U * var)
        mean[s], rstd[s] = mu, r
        tmean[s], trel[s] = em, 0.5 * ev * r * r + 4 * U
        hat = (v - mu.view(1, -1, 1)) * r.view(1, -1, 1)
        zz = hat.reshape(-1, d) * W + B
        eh = (r * em).view(1, -1, 1) + hat.abs() * (trel[s].view(1, -1, 1) + 3 * U)
        z[p:q] = zz
        tz[p:q] = eh.reshape(-1, d) * W.abs() + 3 * U * (zz.abs() + B.abs() + (hat.reshape(-1, d) * W).abs())
    if act == "relu":
        y, ty = z.clamp(min=0), tz
    elif act == "silu":
        y = z * torch.sigmoid(z)
        ty = 1.1 * tz + 16 * U * y.abs()
    else:
        y, ty = z, tz
    return dict(y=y, ty=ty, z=z, tz=tz, mean=mean, rstd=rstd, tmean=tmean, trel=trel, segs=segs)


NORM_ROWS = [  # rows, groups, channels a group
    (1, 1, 1), (5, 1, 8), (3, 4, 2), (7, 16, 1), (64, 1, 47), (33, 3, 12), (1000, 1, 128), (200, 8, 16), (50, 1, 172),
    (9, 2, 256), (20, 1, 1000), (4, 1, 1025), (6, 1, 2048), (3, 2, 1024), (5, 1, 1030), (300, 64, 4), (2, 1000, 2),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_ROWS)))
def test_norm_rows(dtype, case):
    m, groups, cg = NORM_ROWS[case]
    d = groups * cg
    act, out_dtype = ["none", "relu", "silu"][case % 3], [dtype, F32, F16][(case + 1) % 3]
    note(f"group_norm rows {dtype} m={m} groups={groups} cg={cg} {act}")
    x = normal((m, d), dtype, case, 2.0) + normal((d,), dtype, case + 1)
    w, b = (normal((d,), F32, case + 2), normal((d,), F32, case + 3)) if case % 4 else (None, None)
    y, mean, rstd = T.group_norm(x.cuda(), groups, None if w is None else w.cuda(), None if b is None else b.cuda(),
                                 act=act, out_dtype=out_dtype, stats=True)
    ref = norm_reference(x, groups, w, b, None, 1e-5, act)
    close(mean, ref["mean"], ref["tmean"], F32, "mean")
    close(rstd, ref["rstd"], ref["trel"] * ref["rstd"], F32, "rstd")
    close(y, ref["y"], ref["ty"], out_dtype, "y")
    alone = T.group_norm(x.cuda(), groups, None if w is None else w.cuda(), None if b is None else b.cuda(),
                         act=act, out_dtype=out_dtype)
    assert torch.equal(alone, y)


NORM_SEGS = [  # segment sizes, groups, channels a group
    ([1], 1, 1), ([0, 5, 0, 1, 3], 2, 4), ([40, 0, 7, 1, 33], 4, 16), ([300], 1, 40), ([16, 17, 15, 31, 33, 0], 3, 5),
    ([2000, 3, 64, 100], 8, 16), ([5000], 32, 4), ([1] * 200, 1, 128), ([90] * 30 + [700], 1, 172), ([33], 2, 1024),
    ([3] * 1500 + [200, 0, 1], 2, 24), ([70, 80], 1, 1025), ([20_000], 4, 8),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_SEGS)))
def test_norm_segments(dtype, case):
    sizes, groups, cg = NORM_SEGS[case]
    d = groups * cg
    act, out_dtype = ["relu", "none", "silu"][case % 3], [F32, dtype, BF16][case % 3]
    off = ranges(sizes, lead=case % 3)
    m = int(off[-1]) + case % 2
    note(f"group_norm segments {dtype} m={m} segs={len(sizes)} groups={groups} cg={cg} {act}")
    x = normal((m, d), dtype, case, 2.0) + normal((d,), dtype, case + 1)
    x[:case % 3] = float("nan")
    if case % 2:
        x[m - 1] = float("nan")
    w, b = (normal((d,), F32, case + 2), normal((d,), F32, case + 3)) if case % 4 else (None, None)
    out = torch.full((m, d), 9.0, dtype=out_dtype, device="cuda")
    y, mean, rstd = T.group_norm(x.cuda(), groups, None if w is None else w.cuda(), None if b is None else b.cuda(),
                                 off=off.cuda(), act=act, out=out, stats=True)
    ref = norm_reference(x, groups, w, b, off, 1e-5, act)
    filled = torch.tensor(sizes) > 0
    close(mean[filled.cuda()], ref["mean"][filled], ref["tmean"][filled], F32, "mean")
    close(rstd[filled.cuda()], ref["rstd"][filled], (ref["trel"] * ref["rstd"])[filled], F32, "rstd")
    assert (mean.cpu()[~filled] == 0).all() and (rstd.cpu()[~filled] == 0).all()
    r = slice(int(off[0]), int(off[-1]))
    close(y[r], ref["y"][r], ref["ty"][r], out_dtype, "y")
    assert (y[:int(off[0])] == 9.0).all() and (y[int(off[-1]):] == 9.0).all()
    again = T.group_norm(x.cuda(), groups, None if w is None else w.cuda(), None if b is None else b.cuda(),
                         off=off.cuda(), act=act, out_dtype=out_dtype)
    assert torch.equal(again[r], y[r])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("by_seg", [False, True])
def test_norm_strided_and_far_from_zero(dtype, by_seg):
    """Strided and misaligned rows; values far from zero next to their spread
    (a variance taken as a difference of squares would be lost)."""
    note(f"group_norm strided {dtype} segments={by_seg}")
    m, groups, cg = 200, 2, 20
    d = groups * cg
    x = normal((m, d), F32, 1, 0.5) + (1000.0 if dtype != BF16 else 60.0)
    x = x.to(dtype)
    off = ranges([50, 0, 149, 1]) if by_seg else None
    w, b = normal((d,), F32, 2), normal((d,), F32, 3)
    for pad, lead in ((8, 8), (3, 1), (4, 0)):
        wide = torch.full((m, lead + d + pad), 4.0, dtype=dtype, device="cuda")
        out = wide[:, lead:lead + d]
        T.group_norm(strided(x, pad, lead), groups, w.cuda(), b.cuda(), off=None if off is None else off.cuda(), out=out)
        ref = norm_reference(x, groups, w, b, off, 1e-5, "none")
        close(out, ref["y"], ref["ty"], dtype, (pad, lead))
        assert (torch.cat([wide[:, :lead], wide[:, lead + d:]], 1) == 4.0).all()


def test_norm_constant_and_special_rows():
    """Rows without spread come out as the bias; NaN and infinities stay in
    their row or segment."""
    note("group_norm constant and special rows")
    x = torch.full((6, 32), 3.0)
    x[1] = 0.0
    x[3, 5], x[4, 7] = float("nan"), float("inf")
    w, b = normal((32,), F32, 1).cuda(), normal((32,), F32, 2).cuda()
    y = T.group_norm(x.cuda(), 1, w, b).cpu()
    for r in (0, 1, 2, 5):
        assert torch.equal(y[r], b.cpu())
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).any()
    y = T.group_norm(x.cuda(), 1, w, b, off=torch.tensor([0, 1, 3, 4, 5, 6]).cuda()).cpu()
    assert torch.equal(y[0], b.cpu()) and torch.isfinite(y[1:3]).all() and torch.isnan(y[3]).all()
    assert torch.equal(y[5], b.cpu())


def norm_grad_reference(x, dy, groups, w, b, mean, rstd, off, act):
    """Gradients in 64 bits at the given statistics, with tolerances."""
    m, d = x.shape
    cg = d // groups
    W = torch.ones(d).double() if w is None else w.double()
    B = torch.zeros(d).double() if b is None else b.double()
    mean, rstd = mean.double().cpu(), rstd.double().cpu()
    segs = [(r, r + 1) for r in range(m)] if off is None else [(int(p), int(q)) for p, q in zip(off[:-1], off[1:])]
    dx, tdx = torch.zeros(m, d, dtype=torch.float64), torch.zeros(m, d, dtype=torch.float64)
    dw, db, tw, tb = (torch.zeros(d, dtype=torch.float64) for _ in range(4))
    rows = sum(q - p for p, q in segs)
    for s, (p, q) in enumerate(segs):
        if p == q:
            continue
        mu, r = mean[s].view(1, -1, 1), rstd[s].view(1, -1, 1)
        hat = ((x[p:q].double().view(-1, groups, cg) - mu) * r)
        z = hat.reshape(-1, d) * W + B
        y = dy[p:q].double()
        ez = 4 * U * ((hat.reshape(-1, d) * W).abs() + B.abs())
        if act == "relu":
            dz, edz = torch.where(z > 0, y, torch.zeros_like(y)), torch.zeros_like(y)
        elif act == "silu":
            sg = torch.sigmoid(z)
            dz = y * sg * (1 + z * (1 - sg))
            edz = y.abs() * (0.5 * ez + 24 * U)
        else:
            dz, edz = y, torch.zeros_like(y)
        h = hat.reshape(-1, d)
        eh = 3 * U * h.abs()
        dw += (dz * h).sum(0)
        db += dz.sum(0)
        tw += (edz * h.abs() + dz.abs() * eh).sum(0) + (D + 600) * U * (dz * h).abs().sum(0)
        tb += edz.sum(0) + (D + 600) * U * dz.abs().sum(0)
        gz, egz = (dz * W).view(-1, groups, cg), (edz * W.abs() + U * (dz * W).abs()).view(-1, groups, cg)
        s1, s2 = gz.mean((0, 2), keepdim=True), (gz * hat).mean((0, 2), keepdim=True)
        e1 = egz.mean((0, 2), keepdim=True) + D * U * gz.abs().mean((0, 2), keepdim=True)
        e2 = (egz * hat.abs()).mean((0, 2), keepdim=True) + (D + 4) * U * (gz * hat).abs().mean((0, 2), keepdim=True)
        dx[p:q] = (r * (gz - s1 - hat * s2)).reshape(-1, d)
        tdx[p:q] = (r * (egz + e1 + hat.abs() * e2 + 8 * U * (gz.abs() + s1.abs() + (hat * s2).abs()))).reshape(-1, d)
    return dx, tdx, dw, tw, db, tb, rows


def check_norm_grad(x, dy, groups, w, b, off, act, xs=None, ys=None):
    dev = (lambda t: None if t is None else t.cuda())
    xs, ys = dev(x) if xs is None else xs, dev(dy) if ys is None else ys
    _, mean, rstd = T.group_norm(xs, groups, dev(w), dev(b), off=dev(off), act=act, stats=True)
    dx, dw, db = T.group_norm_grad(ys, xs, groups, dev(w), dev(b), mean, rstd, off=dev(off), act=act)
    rdx, tdx, rdw, tw, rdb, tb, _ = norm_grad_reference(x, dy, groups, w, b, mean, rstd, off, act)
    r = slice(0, x.shape[0]) if off is None else slice(int(off[0]), int(off[-1]))
    close(dx[r], rdx[r], tdx[r], x.dtype, "dx")
    close(dw, rdw, tw, F32, "dweight")
    close(db, rdb, tb, F32, "dbias")
    dx2, dw2, db2 = T.group_norm_grad(ys, xs, groups, dev(w), dev(b), mean, rstd, off=dev(off), act=act)
    assert torch.equal(dx[r], dx2[r]) and torch.equal(dw, dw2) and torch.equal(db, db2)
    none, dw3, db3 = T.group_norm_grad(ys, xs, groups, dev(w), dev(b), mean, rstd, off=dev(off), act=act,
                                       need=("weight", "bias"))
    assert none is None and torch.equal(dw, dw3) and torch.equal(db, db3)
    dx4, none, none2 = T.group_norm_grad(ys, xs, groups, dev(w), dev(b), mean, rstd, off=dev(off), act=act,
                                         need=("x",))
    assert none is None and none2 is None and torch.equal(dx[r], dx4[r])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_ROWS)))
def test_norm_rows_grad(dtype, case):
    m, groups, cg = NORM_ROWS[case]
    d = groups * cg
    act = ["relu", "silu", "none"][case % 3]
    note(f"group_norm_grad rows {dtype} m={m} groups={groups} cg={cg} {act}")
    x = normal((m, d), dtype, case, 2.0) + normal((d,), dtype, case + 1)
    w, b = (normal((d,), F32, case + 2), normal((d,), F32, case + 3)) if case % 4 else (None, None)
    check_norm_grad(x, normal((m, d), dtype, case + 4), groups, w, b, None, act)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_SEGS)))
def test_norm_segments_grad(dtype, case):
    sizes, groups, cg = NORM_SEGS[case]
    d = groups * cg
    act = ["silu", "relu", "none"][case % 3]
    off = ranges(sizes, lead=case % 3)
    m = int(off[-1]) + case % 2
    note(f"group_norm_grad segments {dtype} m={m} segs={len(sizes)} groups={groups} cg={cg} {act}")
    x = normal((m, d), dtype, case, 2.0) + normal((d,), dtype, case + 1)
    dy = normal((m, d), dtype, case + 4)
    for t in (x, dy):
        t[:case % 3] = float("nan")
        if case % 2:
            t[m - 1] = float("nan")
    w, b = (normal((d,), F32, case + 2), normal((d,), F32, case + 3)) if case % 4 else (None, None)
    xs, ys = (strided(x, 3, 1), strided(dy, 8, 0)) if case % 2 else (None, None)
    check_norm_grad(x, dy, groups, w, b, off, act, xs, ys)


@pytest.mark.parametrize("by_seg", [False, True])
def test_norm_grad_without_rows(by_seg):
    note(f"group_norm_grad without rows, segments={by_seg}")
    x = torch.empty(0, 16, device="cuda")
    for segs in ([0] if not by_seg else [0, 3]):
        off = torch.zeros(segs + 1, dtype=torch.int64, device="cuda") if by_seg else None
        y, mean, rstd = T.group_norm(x, 4, off=off, stats=True)
        assert tuple(y.shape) == (0, 16) and tuple(mean.shape) == (segs, 4) and not rstd.any()
        dx, dw, db = T.group_norm_grad(x, x, 4, None, None, mean, rstd, off=off)
        assert tuple(dx.shape) == (0, 16) and not dw.any() and not db.any()
    if by_seg:  # rows, but no segment holds any
        x = torch.ones(5, 16, device="cuda")
        off = torch.zeros(1, dtype=torch.int64, device="cuda")
        y, mean, rstd = T.group_norm(x, 4, off=off, stats=True)
        _, dw, db = T.group_norm_grad(x, x, 4, None, None, mean, rstd, off=off)
        assert not dw.any() and not db.any()


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("off", [None, [0, 11, 11, 40]])
def test_norm_differences(act, off):
    """Gradients against central differences of the 64-bit definition; the
    third derivatives along v are below 1e3 here, h^2 / 6 of that is 1.7e-6."""
    note(f"group_norm differences {act} {off}")
    m, groups, cg = 40, 2, 6
    d = groups * cg
    off_t = None if off is None else torch.tensor(off)
    x, w, b, c = normal((m, d), F32, 1), normal((d,), F32, 2), normal((d,), F32, 3), normal((m, d), F32, 4)
    _, mean, rstd = T.group_norm(x.cuda(), groups, w.cuda(), b.cuda(), off=None if off is None else off_t.cuda(),
                                 act=act, stats=True)
    grads = T.group_norm_grad(c.cuda(), x.cuda(), groups, w.cuda(), b.cuda(), mean, rstd,
                              off=None if off is None else off_t.cuda(), act=act)

    def loss(x, w, b):
        return float((norm_reference(x, groups, w, b, off_t, 1e-5, act)["y"] * c.double()).sum())
    at = [x.double(), w.double(), b.double()]
    for which, grad in enumerate(grads):
        v = normal(tuple(grad.shape), F32, 20 + which).double()
        v = v / v.norm()
        h = 1e-4
        hi, lo = list(at), list(at)
        hi[which], lo[which] = at[which] + h * v, at[which] - h * v
        diff = (loss(*hi) - loss(*lo)) / (2 * h)
        got = float((grad.double().cpu() * v).sum())
        size = float((grad.double().cpu().abs() * v.abs()).sum())
        assert abs(got - diff) <= 2 * D * U * (size + 10) + 2e-6 * (1 + abs(diff)), (which, got, diff)


def test_relu_border_is_exact():
    """Arguments within rounding of ReLU's border: the side is the exact one."""
    note("group_norm_grad relu border")
    m, d = 4096, 64
    x = normal((m, d), F32, 1)
    _, mean, rstd = T.group_norm(x.cuda(), 1, stats=True)
    w = torch.ones(d)
    # the bias takes row 7's values to the border, within one rounding
    hat = (x.double() - mean.double().cpu()) * rstd.double().cpu()
    b = (-hat[7]).float()
    x = x[7:8].expand(m, d).contiguous()
    x = x * (1 + 2.0 ** -23 * torch.randint(-2, 3, (m, d), generator=torch.Generator().manual_seed(3)))
    mean, rstd = mean[7:8].expand(m, 1).contiguous(), rstd[7:8].expand(m, 1).contiguous()
    dy = torch.ones(m, d)
    for off in (None, torch.arange(0, m + 1, 16)):
        mu, rs = (mean, rstd) if off is None else (mean[:m // 16].contiguous(), rstd[:m // 16].contiguous())
        _, _, db = T.group_norm_grad(dy.cuda(), x.cuda(), 1, w.cuda(), b.cuda(), mu, rs, act="relu",
                                     off=None if off is None else off.cuda())
        z = (x.double() - mean.double().cpu()) * rstd.double().cpu() + b.double()
        assert torch.equal(db.cpu().double(), (z > 0).double().sum(0))


@pytest.mark.parametrize("m", [1, 5, 63, 64, 500])
def test_norm_grad_of_no_segments_writes_zeros(m):
    """No segment holds a row: the weights' gradients are zeros, written also
    where the call needs no workspace."""
    note(f"group_norm_grad of no segments m={m}")
    L, x, off = N.lib(), torch.ones(m, 16, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    dw, db = (torch.full((16,), float("nan"), device="cuda") for _ in range(2))
    nbytes = L.taurus_group_norm_bytes(N.F32, m, 16, 4, 0, 1, 1)
    work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    N.check(L.taurus_group_norm_grad(x.data_ptr(), 16, x.data_ptr(), 16, N.F32, m, 16, 4, off.data_ptr(), 0, None, None,
                                     None, None, N.ACT_NONE, None, 16, dw.data_ptr(), db.data_ptr(),
                                     work.data_ptr() if nbytes else None, nbytes,
                                     torch.cuda.current_stream().cuda_stream), "taurus_group_norm_grad")
    assert (dw == 0).all() and (db == 0).all()


SILU_AT = [0.0, 1e-30, -1e-30, 0.5, -0.5, 1.0, -1.0, 8.0, -8.0, 17.0, -17.0, 60.0, -60.0, 87.0, -87.0, 87.6, -87.6, 88.5,
           -88.5, 95.0, -95.0, 200.0, -200.0, 1e30, -1e30, 2.5e38, -2.5e38, 3.4e38, -3.4e38, float("inf"), -float("inf")]


@pytest.mark.parametrize("off", [None, [0, 3]])
def test_silu_at_any_argument(off):
    """With weights of zero the argument is the bias.  The sigmoid q is within
    8 U of itself (power of two, sum, reciprocal, each rounded); under
    z = -87.3 it passes below the least normal fp32 value 2^-126 and may be 0,
    so that z q is off by less than 89 x 2^-126 < 2^-119.  The slope
    q (1 + z (1 - q)) varies with q by at most 1 + |z|, from z = 20 on not at
    all: there q is 1.  Both have limits at infinity: z and 1, 0 and 0."""
    note(f"silu at any argument {off}")
    z = torch.tensor(SILU_AT)
    d, m = z.numel(), 3
    x, zero = normal((m, d), F32, 1).cuda(), torch.zeros(d, device="cuda")
    off = None if off is None else torch.tensor(off, device="cuda")
    y, mean, rstd = T.group_norm(x, 1, zero, z.cuda(), off=off, act="silu", stats=True)
    dx, dw, db = T.group_norm_grad(torch.ones_like(x), x, 1, zero, z.cuda(), mean, rstd, off=off, act="silu")
    zd = z.double().clamp(-1e300, 1e300)
    q = torch.sigmoid(zd)
    ref, slope = zd * q, q * (1 + zd * (1 - q))
    top = torch.isinf(z) & (z > 0)
    assert (y.cpu()[:, top] == float("inf")).all()
    near = 16 * U * ref[~top].abs() + 2.0 ** -119
    for r in range(m):
        close(y[r][~top.cuda()], ref[~top], near, F32, "silu")
    close(db, m * slope, m * (8 * U * q * (1 + zd.abs().clamp(max=20)) + 8 * U * slope.abs() + 2.0 ** -119), F32, "slope")
    assert (dx == 0).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("off", [None, [0, 40]])
def test_silu_of_arguments_past_fp32(off):
    """Arguments that overflow fp32 to infinity: z above, 0 below."""
    note(f"silu past fp32 {off}")
    x = normal((40, 16), F32, 1)
    w = torch.full((16,), 3e38)
    y = T.group_norm(x.cuda(), 1, w.cuda(), off=None if off is None else torch.tensor(off, device="cuda"), act="silu").cpu()
    z = norm_reference(x, 1, w, None, None if off is None else torch.tensor(off), 1e-5, "none")["z"]
    assert (y[z > 4e38] == float("inf")).all() and (y[z < -1e3] == 0).all() and not torch.isnan(y).any()
    assert (z > 4e38).any() and (z < -4e38).any()


@pytest.mark.parametrize("sizes", [[40], [300], [3] * 30])
@pytest.mark.parametrize("scale", [1e-20, 1e-12, 1e12])
def test_norm_grad_of_any_spread(sizes, scale):
    """rstd from 1e-12 to 1e20 (eps may be 0): its square alone passes fp32."""
    note(f"group_norm_grad spread {scale} {sizes[:3]}")
    off, groups, d = ranges(sizes), 2, 24
    m = int(off[-1])
    x = normal((m, d), F32, 1, scale)
    w, b, dy = normal((d,), F32, 2), normal((d,), F32, 3), normal((m, d), F32, 4)
    ref = norm_reference(x, groups, w, b, off, 0.0, "none")
    mean, rstd = ref["mean"].float(), ref["rstd"].float()
    for o, mu, rs in ((off, mean, rstd), (None, mean.repeat_interleave(torch.tensor(sizes), 0),
                                          rstd.repeat_interleave(torch.tensor(sizes), 0))):
        dx, dw, db = T.group_norm_grad(dy.cuda(), x.cuda(), groups, w.cuda(), b.cuda(), mu.cuda(), rs.cuda(),
                                       off=None if o is None else o.cuda())
        rdx, tdx, rdw, tw, rdb, tb, _ = norm_grad_reference(x, dy, groups, w, b, mu, rs, o, "none")
        close(dx, rdx, tdx, F32, "dx")
        close(dw, rdw, tw, F32, "dweight")
        close(db, rdb, tb, F32, "dbias")


# ---------------------------------------------- norms held to their own sums --

def norm_vectors(dtype, cg):
    """Values of a vector, and vectors, of a group of cg channels."""
    e = next(v for v in ([4, 1] if dtype == F32 else [8, 4, 1]) if cg >= v)
    return e, -(-cg // e)


def norm_truth(x, groups, w, b, off, eps, act):
    """Group norm in 64 bits on the device, every segment at once, with
    tolerances from the additions that a value passes.

    A row by itself: a lane adds its values, at most 16, one after another;
    the lanes of a wave join in 6 steps, of four waves in 2 more.  Segments:
    a thread adds up to eight rows of a vector in four chains of at most 16,
    joins them, and joins what it has of one batch of rows after another
    (four roundings each); then up to 64 lanes go through a group's threads,
    and a long segment's units are added by a wave or four.  A mean is off by
    the additions' depth, the squares by theirs and, where means of parts
    are joined, by twice the means' error times the spread."""
    x = x.cuda()
    m, d = x.shape
    cg = d // groups
    e, cgv = norm_vectors(x.dtype, cg)
    xd = x.double()
    W = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double().cuda()
    B = torch.zeros(d, dtype=torch.float64, device="cuda") if b is None else b.double().cuda()
    if off is None:
        seg, count = torch.arange(m, device="cuda"), torch.ones(m, dtype=torch.int64, device="cuda")
        first, end = 0, m
    else:
        first, end = int(off[0]), int(off[-1])
        count = (off[1:] - off[:-1]).cuda()
        seg = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count)
    xg = xd[first:end].view(-1, groups, cg)

    def per_segment(v):  # sums of [rows][groups] over a segment's rows
        return torch.zeros(count.numel(), groups, dtype=torch.float64, device="cuda").index_add_(0, seg, v)
    size = (count.clamp(min=1) * cg).double().unsqueeze(1)
    mean = per_segment(xg.sum(2)) / size
    var = per_segment(((xg - mean[seg].unsqueeze(2)) ** 2).sum(2)) / size
    rstd = (var + eps) ** -0.5
    sizes = per_segment(xg.abs().sum(2)) / size
    top = torch.zeros(count.numel(), groups, dtype=torch.float64, device="cuda")
    top.scatter_reduce_(0, seg.unsqueeze(1).expand(-1, groups), xg.abs().amax(2), "amax")
    nv = groups * cgv
    longest = int(count.max()) if count.numel() else 0
    if off is None:
        depth = min(cg, 16) + 6 + 2
        em = (depth + 3) * U * sizes
        ev = (depth + 5) * U * var + em ** 2
    else:
        ry = max(1, (64 if nv <= 64 else 256) // nv)          # rows side by side, at least
        rows = min(longest, 4096)                             # of a unit, at most
        batches = -(-rows // (4 * ry))
        joins = -(-(min(ry if nv <= 64 else 256 // min(nv, 256), rows) * 4 * cgv) // 64) + 6
        units = 0 if longest <= 64 else -(-(-(-longest // 64)) // 64) + 8
        em = U * (16 + 3) * sizes + U * (4 * (batches - 1) + 2 * (joins + 3) + 2 * (units + 3) * (units > 0)) * top
        ev = (16 + 4 * batches + joins + units + 12) * U * var + 4 * em * var.sqrt() + 4 * em ** 2
    trel = 0.5 * (ev + U * (var + eps)) * rstd ** 2 + 5 * U
    hat = (xg - mean[seg].unsqueeze(2)) * rstd[seg].unsqueeze(2)
    eh = (rstd * em)[seg].unsqueeze(2) + hat.abs() * (trel[seg].unsqueeze(2) + 3 * U)
    t = hat.reshape(-1, d) * W
    z, tz = t + B, eh.reshape(-1, d) * W.abs()
    tz = tz + 3 * U * (z.abs() + B.abs() + t.abs())
    if act == "relu":
        y, ty = z.clamp(min=0), tz
    elif act == "silu":
        y = z * torch.sigmoid(z)
        ty = 1.1 * tz + 16 * U * y.abs()
    else:
        y, ty = z, tz
    return dict(y=y, ty=ty, mean=mean, em=em, rstd=rstd, trel=trel, seg=seg, count=count, rows=slice(first, end), nv=nv,
                longest=longest)


def norm_grad_truth(x, dy, groups, w, b, mean, rstd, off, act, ref):
    """The gradients at the given statistics, likewise."""
    x, dy = x.cuda(), dy.cuda()
    m, d = x.shape
    cg = d // groups
    e, cgv = norm_vectors(x.dtype, cg)
    seg, count, r = ref["seg"], ref["count"], ref["rows"]
    W = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double().cuda()
    B = torch.zeros(d, dtype=torch.float64, device="cuda") if b is None else b.double().cuda()
    mu, rs = mean.double()[seg].unsqueeze(2), rstd.double()[seg].unsqueeze(2)
    hat = (x[r].double().view(-1, groups, cg) - mu) * rs
    h, y = hat.reshape(-1, d), dy[r].double()
    z = h * W + B
    ez = 4 * U * ((h * W).abs() + B.abs())
    if act == "relu":
        dz, edz = torch.where(z > 0, y, 0.0), torch.zeros_like(y)
    elif act == "silu":
        q = torch.sigmoid(z)
        dz = y * q * (1 + z * (1 - q))
        edz = y.abs() * (0.5 * ez + 8 * U * q * (1 + z.abs().clamp(max=20)) + 8 * U)
    else:
        dz, edz = y, torch.zeros_like(y)
    nv, longest = ref["nv"], ref["longest"]
    if off is None:
        lanes = min(64, 1 << max(0, (cgv - 1).bit_length())) if cg <= 1024 else 256
        per = 256 // lanes
        depth = min(cg, 16) + 6 + 2
        blocks = min(-(-m * groups // (8 * per)), 1024)
        column = -(-m * groups // max(1, (blocks * per // groups) * groups)) + -(-blocks * per // groups // 64) + 20
    else:
        wave = nv <= 64
        ry, ry_most = max(1, (64 if wave else 256) // nv), max(1, 256 // nv)
        rows = -(-min(longest, 4096) // ry)                   # a thread's of a unit
        slots = -(-(m // 64 + count.numel()) // 4096)         # a workgroup's
        joins = -(-(min(ry_most, longest) * cgv) // 64) + 6
        units = 0 if longest <= 64 else -(-(-(-longest // 64)) // 64) + 8
        depth = rows + e + joins + units
        column = slots * rows + ry_most + 64 + 20
    eh = 3 * U * h.abs()
    dw, db = (dz * h).sum(0), dz.sum(0)
    tw = (edz * h.abs() + dz.abs() * eh).sum(0) + (column + 4) * U * (dz * h).abs().sum(0)
    tb = edz.sum(0) + column * U * dz.abs().sum(0)
    gz, egz = (dz * W).view(-1, groups, cg), (edz * W.abs() + U * (dz * W).abs()).view(-1, groups, cg)

    def averages(v):
        total = torch.zeros(count.numel(), groups, dtype=torch.float64, device="cuda").index_add_(0, seg, v.sum(2))
        return (total / (count.clamp(min=1) * cg).double().unsqueeze(1))[seg].unsqueeze(2)
    s1, s2 = averages(gz), averages(gz * hat)
    e1 = averages(egz) + (depth + 3) * U * averages(gz.abs())
    e2 = averages(egz * hat.abs()) + (depth + 7) * U * averages((gz * hat).abs())
    dx = (rs * (gz - s1 - hat * s2)).reshape(-1, d)
    tdx = (rs * (egz + e1 + hat.abs() * e2 + 8 * U * (gz.abs() + s1.abs() + (hat * s2).abs()))).reshape(-1, d)
    return dx, tdx, dw, tw, db, tb


def near(got, ref, tol, dtype, what):
    """close, on the device."""
    got = got.double()
    bound = tol + HALF[dtype] * (ref.abs() + tol) + TINY[dtype]
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / bound)[bad].max()), bad.nonzero()[:4].tolist())


def check_norm(x, dy, groups, w, b, off, act):
    """Forward and gradients against the 64-bit forms; rows outside stay."""
    d = x.shape[1]
    dev = (lambda t: None if t is None else t.cuda())
    xs, ys, wd, bd, od = x.cuda(), dy.cuda(), dev(w), dev(b), dev(off)
    ref = norm_truth(x, groups, w, b, off, 1e-5, act)
    r = ref["rows"]
    out = torch.full_like(xs, 9.0)
    y, mean, rstd = T.group_norm(xs, groups, wd, bd, off=od, act=act, out=out, stats=True)
    held = ref["count"] > 0
    near(mean[held], ref["mean"][held], ref["em"][held], F32, "mean")
    near(rstd[held], ref["rstd"][held], (ref["trel"] * ref["rstd"])[held], F32, "rstd")
    assert (mean[~held] == 0).all() and (rstd[~held] == 0).all()
    near(y[r], ref["y"], ref["ty"], x.dtype, "y")
    assert (y[:r.start] == 9.0).all() and (y[r.stop:] == 9.0).all()
    dx, dw, db = T.group_norm_grad(ys, xs, groups, wd, bd, mean, rstd, off=od, act=act)
    rdx, tdx, rdw, tw, rdb, tb = norm_grad_truth(x, dy, groups, w, b, mean, rstd, off, act, ref)
    near(dx[r], rdx, tdx, x.dtype, "dx")
    near(dw, rdw, tw, F32, "dweight")
    near(db, rdb, tb, F32, "dbias")
    again = T.group_norm_grad(ys, xs, groups, wd, bd, mean, rstd, off=od, act=act)
    assert torch.equal(again[0][r], dx[r]) and torch.equal(again[1], dw) and torch.equal(again[2], db)


def norm_inputs(m, d, dtype, seed):
    x = normal((m, d), dtype, seed, 2.0) + normal((d,), dtype, seed + 1)
    return x, normal((m, d), dtype, seed + 2), normal((d,), F32, seed + 3), normal((d,), F32, seed + 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_ROWS)))
def test_norm_rows_held_to_their_depth(dtype, case):
    m, groups, cg = NORM_ROWS[case]
    note(f"group_norm depth rows {dtype} m={m} groups={groups} cg={cg}")
    x, dy, w, b = norm_inputs(m, groups * cg, dtype, case)
    check_norm(x, dy, groups, w, b, None, ["silu", "none", "relu"][case % 3])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(NORM_SEGS)))
def test_norm_segments_held_to_their_depth(dtype, case):
    sizes, groups, cg = NORM_SEGS[case]
    note(f"group_norm depth segments {dtype} segs={len(sizes)} groups={groups} cg={cg}")
    off = ranges(sizes)
    x, dy, w, b = norm_inputs(int(off[-1]), groups * cg, dtype, case)
    check_norm(x, dy, groups, w, b, off, ["none", "relu", "silu"][case % 3])


def segment_sizes(count, sizes, long, seed):
    """count segments of the given sizes, a few long ones among them."""
    g = torch.Generator().manual_seed(seed)
    s = torch.tensor(sizes)[torch.randint(0, len(sizes), (count,), generator=g)]
    s[torch.randperm(count, generator=g)[:len(long)]] = torch.tensor(long, dtype=torch.int64)
    return s.tolist()


MANY = [  # segments, sizes, long ones, groups, channels a group
    (9_000, [0, 0, 1, 2, 3, 5, 30], [129, 200, 256, 257, 400] * 20, 2, 12),    # a wave a slot, several slots each
    (9_000, [0, 1, 7, 63, 64, 65], [], 1, 5),
    (5_000, [0, 1, 2, 5, 9], [300, 1000, 77], 4, 160),                         # four waves a slot
    (4_300, [0, 1, 1, 2], [90, 65], 1, 2048),                                  # rows wider than a workgroup
    (24, [200, 130, 90, 65], [], 64, 4),                                       # 1,536 joins
    (1_023, [130, 90, 200], [], 2, 8),                                         # 2,046 joins of a few units each
    (3, [1], [70_000, 200_000, 30_000], 2, 8),                                 # units of 128 rows
    (2, [600_000], [], 1, 8),                                                  # units of 512 rows
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(MANY)))
def test_norm_of_many_and_long_segments(dtype, case):
    """More slots than workgroups, more joins than 1,024, longer units."""
    count, sizes, long, groups, cg = MANY[case]
    off = ranges(segment_sizes(count, sizes, long, case), lead=5)
    m = int(off[-1]) + 3
    note(f"group_norm many {dtype} m={m} segs={count} groups={groups} cg={cg}")
    x, dy, w, b = norm_inputs(m, groups * cg, dtype, case)
    for t in (x, dy):
        t[:5], t[m - 3:] = float("nan"), float("nan")
    check_norm(x, dy, groups, w, b, off, ["relu", "silu", "none"][case % 3])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,groups,cg", [(140_001, 1, 64), (9_001, 1, 2048), (30_011, 40, 5), (1_100_003, 1, 7)])
def test_norm_of_many_rows(dtype, m, groups, cg):
    """More rows than the launch has lanes for: each takes several."""
    note(f"group_norm many rows {dtype} m={m} groups={groups} cg={cg}")
    x, dy, w, b = norm_inputs(m, groups * cg, dtype, 3)
    check_norm(x, dy, groups, w, b, None, "silu")


# ------------------------------------------------- streams, graphs, refusals --

def everything(t):
    """One pass of every operator over the tensors of `t`."""
    h = T.lookup_rows(t["table"], t["ids"], 1.5)
    z = T.grouped_linear(h, t["off"], t["weight"], t["bias"])
    y, mean, rstd = T.group_norm(z, 4, t["gamma"], t["beta"], act="silu", stats=True)
    q, mean2, rstd2 = T.group_norm(z, 2, t["gamma"], t["beta"], off=t["off"], act="relu", stats=True)
    dz, dgamma, dbeta = T.group_norm_grad(y, z, 4, t["gamma"], t["beta"], mean, rstd, act="silu")
    dz2, dgamma2, dbeta2 = T.group_norm_grad(q, z, 2, t["gamma"], t["beta"], mean2, rstd2, off=t["off"], act="relu")
    dh, dw, db = T.grouped_linear_grad(dz, h, t["off"], t["weight"])
    dt = T.lookup_rows_grad(dh, t["ids"], t["table"].shape[0], 1.5)
    return [h, z, y, mean, rstd, q, mean2, rstd2, dz, dgamma, dbeta, dz2, dgamma2, dbeta2, dh, dw, db, dt]


def everything_inputs(seed, dtype=BF16, m=5000, n=700, k=64, c=48):
    off = ranges([m // 2, 0, m // 8, m - m // 2 - m // 8])
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(-1, n, (m,), generator=g, dtype=torch.int32)
    t = dict(table=normal((n, k), dtype, seed), ids=ids, off=off, weight=normal((4, k, c), dtype, seed + 1, 0.1),
             bias=normal((4, c), F32, seed + 2), gamma=normal((c,), F32, seed + 3), beta=normal((c,), F32, seed + 4))
    return {k: v.cuda() for k, v in t.items()}


@pytest.mark.parametrize("dtype", DTYPES)
def test_graph_replays(dtype):
    """A captured pass replays with new inputs, between eager work."""
    note(f"graph {dtype}")
    t = everything_inputs(1, dtype)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        everything(t)
    torch.cuda.current_stream().wait_stream(s)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(t)
    with torch.cuda.graph(second):  # two graphs' workspaces are their own
        outs2 = everything(t)
    for seed in (1, 2, 3, 4):
        for key, v in everything_inputs(seed, dtype).items():
            t[key].copy_(v)
        want = everything(t)
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        for i, (a, b, c) in enumerate(zip(outs, outs2, want)):
            assert torch.equal(a, c) and torch.equal(b, c), (seed, i)


def test_far_rows():
    """Rows far apart in arrays of 2.6e9 values, past what 32 bits hold:
    linear maps and norms give the dense rows' bits."""
    note("far rows")
    m, apart, k, n = 40_001, 65_600, 64, 72

    def far(width):
        return torch.empty(m * apart, dtype=BF16, device="cuda").view(m, apart)[:, :width]
    off = ranges([12_000, 0, 1, m - 12_001]).cuda()
    x, dy = normal((m, k), BF16, 1).cuda(), normal((m, n), BF16, 2).cuda()
    w = normal((4, k, n), BF16, 3, k ** -0.5).cuda()
    fx, fdy, out = far(k), far(n), far(n)
    fx.copy_(x)
    fdy.copy_(dy)
    T.grouped_linear(fx, off, w, out=out)
    y = T.grouped_linear(x, off, w)
    assert torch.equal(out, y)
    for got, want in zip(T.grouped_linear_grad(fdy, fx, off, w), T.grouped_linear_grad(dy, x, off, w)):
        assert torch.equal(got, want)
    for o in (None, off):
        _, mean, rstd = T.group_norm(dy, 4, off=o, act="silu", stats=True)
        want = T.group_norm(dy, 4, off=o, act="silu")
        assert torch.equal(T.group_norm(fdy, 4, off=o, act="silu", out=out), want)
        for got, ref in zip(T.group_norm_grad(out, fdy, 4, None, None, mean, rstd, off=o, act="silu"),
                            T.group_norm_grad(want, dy, 4, None, None, mean, rstd, off=o, act="silu")):
            assert torch.equal(got, ref)


def test_streams():
    """Two streams at once, and the stream argument, give the eager bits."""
    note("streams")
    t, u = everything_inputs(1), everything_inputs(2, m=30_000)
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
    h = T.lookup_rows(t["table"], t["ids"], 1.5, stream=a)
    z = T.grouped_linear(h, t["off"], t["weight"], t["bias"], stream=a)
    y, mean, rstd = T.group_norm(z, 4, t["gamma"], t["beta"], act="silu", stats=True, stream=a)
    dz, _, _ = T.group_norm_grad(y, z, 4, t["gamma"], t["beta"], mean, rstd, act="silu", stream=a)
    dh, dw, _ = T.grouped_linear_grad(dz, h, t["off"], t["weight"], stream=a)
    dt = T.lookup_rows_grad(dh, t["ids"], 700, 1.5, stream=a)
    a.synchronize()
    for x, y in zip([h, z, dz, dh, dw, dt], [want[0], want[1], want[8], want[14], want[15], want[17]]):
        assert torch.equal(x, y)


def test_wrapper_refusals():
    note("refusals")
    x = torch.zeros(8, 16, device="cuda")
    ids = torch.zeros(8, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 8], device="cuda")
    w = torch.zeros(1, 16, 16, device="cuda")
    v = torch.zeros(16, device="cuda")
    st = torch.zeros(8, 1, device="cuda")
    bad = [
        lambda: T.lookup_rows(x, ids.long()), lambda: T.lookup_rows(x, ids.cpu()), lambda: T.lookup_rows(x.double(), ids),
        lambda: T.lookup_rows(x, ids, out=x), lambda: T.lookup_rows(x[0], ids), lambda: T.lookup_rows(x, ids[::2]),
        lambda: T.lookup_rows(x, ids, out=torch.empty(7, 16, device="cuda")), lambda: T.lookup_rows(x.t(), ids),
        lambda: T.lookup_rows(x, ids, out=torch.empty(8, 16, device="cuda"), out_dtype=BF16),
        lambda: T.lookup_rows_grad(x[:1].expand(8, 16), ids, 9), lambda: T.lookup_rows_grad(x, ids[:7], 9),
        lambda: T.lookup_rows_grad(x, ids, 8, out=x), lambda: T.lookup_rows_grad(x, ids, 8, out=x[:, :16]),
        lambda: T.grouped_linear(x, off.int(), w), lambda: T.grouped_linear(x, off, w.to(BF16)),
        lambda: T.grouped_linear(x, off, w[0]), lambda: T.grouped_linear(x, off, w.transpose(1, 2)),
        lambda: T.grouped_linear(x, off, torch.zeros(2, 16, 16, device="cuda")),
        lambda: T.grouped_linear(x, off, w, torch.zeros(1, 15, device="cuda")),
        lambda: T.grouped_linear(x, off, w, torch.zeros(1, 16, device="cuda", dtype=BF16)),
        lambda: T.grouped_linear(x, off, w, out=x), lambda: T.grouped_linear_grad(x.to(BF16), x, off, w),
        lambda: T.grouped_linear_grad(x[:, :8], x, off, w),
        lambda: T.grouped_linear_grad(x, x, off, w, weight_dtype=torch.float64),
        lambda: T.group_norm(x, 1, v.to(BF16)), lambda: T.group_norm(x, 1, v[:15]), lambda: T.group_norm(x, act="gelu"),
        lambda: T.group_norm(x, off=off.int()), lambda: T.group_norm(x, out=x),
        lambda: T.group_norm_grad(x, x, 1, v, v, st[:7], st), lambda: T.group_norm_grad(x, x, 2, v, v, st, st),
        lambda: T.group_norm_grad(x, x, 1, v, v, st, st.double()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted", i)
    for call in (lambda: T.group_norm(x, 3), lambda: T.group_norm(x, 0),
                 lambda: T.group_norm(x, eps=-1.0), lambda: T.group_norm(torch.zeros(2, 4096, device="cuda"))):
        with pytest.raises(T.TaurusError):
            call()
    # columns of one wide array do not overlap
    wide = torch.zeros(8, 32, device="cuda")
    T.group_norm(wide[:, :16], out=wide[:, 16:])
    T.grouped_linear(wide[:, 16:], off, w, out=wide[:, :16])


def test_broken_offsets_touch_nothing_else():
    """Offsets outside [0, m] are clamped: rows around the arrays stay."""
    note("offsets outside the rows")
    for dtype in (F32, BF16):
        big = torch.full((300, 16), 2.0, dtype=dtype, device="cuda")
        x = torch.ones(100, 16, dtype=dtype, device="cuda")
        w = torch.ones(3, 16, 16, dtype=dtype, device="cuda")
        off = torch.tensor([-50, 40, 10_000, 2 ** 40], device="cuda")
        T.grouped_linear(x, off, w, out=big[100:200])
        assert (big[:100] == 2).all() and (big[200:] == 2).all() and (big[100:200] == 16).all()
        T.group_norm(x, off=off, out=big[100:200])
        assert (big[:100] == 2).all() and (big[200:] == 2).all() and (big[100:200] == 0).all()
        back = torch.tensor([60, 20, 90, 5], device="cuda")
        T.grouped_linear(x, back, w, out=big[100:200])
        T.group_norm(x, off=back, out=big[100:200])
        _, dw, _ = T.grouped_linear_grad(x, x, back, w)
        assert (big[:100] == 2).all() and (big[200:] == 2).all()


# ------------------------------------------------------------- together --

def test_encoder_and_norms_in_a_model():
    """Learned rows by id, a linear map per vertex type and a norm make a
    GraphSAGE model's input; its hidden layer is normalised; against the
    same model in 64 bits."""
    from fixtures import workloads as WL
    from tests import harness as H
    note("encoder and norms in a model")
    n = WL.SAGE_RMAT_4K.n
    src, dst = WL.graph(WL.SAGE_RMAT_4K)
    row_off, col_dst = T.build_csr(n, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda())
    sizes = [n // 2, 0, n // 3, n - n // 2 - n // 3]
    off = ranges(sizes)
    table, rows = normal((500, 24), F32, 1), 500
    ids = torch.randint(0, rows, (n,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    w, b = normal((4, 24, 32), F32, 3, 0.2), normal((4, 32), F32, 4)
    g1, b1, g2, b2 = (normal((d,), F32, s) for d, s in ((32, 5), (32, 6), (16, 7), (16, 8)))
    wc1, wc2 = normal((32, 32), F32, 9, 0.2).numpy(), normal((16, 16), F32, 10, 0.2).numpy()
    bias1, bias2 = normal((16,), F32, 11).numpy(), normal((8,), F32, 12).numpy()
    layers = [dict(agg=N.SAGE_MEAN, d_in=32, d_out=16, weight_cat=wc1, bias=bias1, relu=False, layer=1,
                   norm=dict(groups=2, weight=g2.cuda(), bias=b2.cuda(), act="relu")),
              dict(agg=N.SAGE_MEAN, d_in=16, d_out=8, weight_cat=wc2, bias=bias2, relu=False, layer=2)]
    enc = dict(ids=ids.cuda(), scale=2.0, off=off.cuda(), weight=w.cuda(), bias=b.cuda(),
               norm=dict(groups=1, weight=g1.cuda(), bias=b1.cuda(), act="silu"))
    outs, _ = T.run_layers(n, row_off, col_dst, table.cuda(), layers, chunk=1024, encoder=enc)

    def sage(h, wc, bias):
        d_out = wc.shape[1] // 2
        W = torch.from_numpy(wc).double()
        s = torch.zeros(n, h.shape[1], dtype=torch.float64)
        s.index_add_(0, torch.from_numpy(dst).long(), h[torch.from_numpy(src).long()])
        deg = torch.bincount(torch.from_numpy(dst).long(), minlength=n).clamp(min=1).double().unsqueeze(1)
        return (s / deg) @ W[:, :d_out] + h @ W[:, d_out:] + torch.from_numpy(bias).double()
    at = torch.repeat_interleave(torch.arange(4), torch.tensor(sizes))
    h = table.double()[ids.long()] * 2.0
    h = torch.bmm(h.unsqueeze(1), w.double()[at]).squeeze(1) + b.double()[at]
    h = norm_reference(h, 1, g1, b1, None, 1e-5, "silu")["y"]
    z1 = norm_reference(sage(h, wc1, bias1), 2, g2, b2, None, 1e-5, "relu")["y"]
    z2 = sage(z1, wc2, bias2)
    for got, ref in zip(outs, (z1, z2)):
        r = H.compare(got.cpu().numpy(), ref.numpy(), H.RTOL[N.F32])
        assert r["n_bad"] == 0, r
    given = [torch.empty_like(o) for o in outs]
    again, _ = T.run_layers(n, row_off, col_dst, table.cuda(), layers, chunk=1024, encoder=enc, outs=given)
    for a, g, o in zip(again, given, outs):
        assert a is g and torch.equal(a, o)
    with pytest.raises(ValueError, match="does not know"):
        T.run_layers(n, row_off, col_dst, table.cuda(), layers, chunk=1024, encoder=dict(enc, foo=1))
    with pytest.raises(ValueError, match="together"):
        T.run_layers(n, row_off, col_dst, table.cuda(), layers, chunk=1024, encoder=dict(weight=w.cuda()))


def test_model_on_a_stream_of_its_own():
    """A model whose last layer is normalised, run on another stream than the
    current one, is complete when it returns and gives the same bits."""
    note("model on a stream of its own")
    n, d = 200_003, 64
    src = torch.arange(n).repeat(4)
    dst = (src + torch.tensor([1, 77, 5_003, 100_001]).repeat_interleave(n)) % n
    row_off, col_dst = T.build_csr(n, src.int().cuda(), dst.int().cuda())
    x = normal((n, d), F32, 2).cuda()
    off = torch.arange(0, n + 1, n // 7).cuda()
    off[-1] = n
    layers = [dict(agg=N.SAGE_MEAN, d_in=d, d_out=d, weight_cat=normal((d, 2 * d), F32, 3, 0.2).numpy(), bias=None,
                   layer=i + 1, norm=dict(groups=4, off=off, act="silu")) for i in range(2)]
    enc = dict(norm=dict(groups=1, act="relu"))
    want, _ = T.run_layers(n, row_off, col_dst, x, layers, chunk=65536, encoder=enc)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, _ = T.run_layers(n, row_off, col_dst, x, layers, chunk=65536, encoder=enc, stream=s)
    here = [a.clone() for a in got]  # on the current stream, which waits for nothing
    for a, b in zip(here, want):
        assert torch.equal(a, b)
