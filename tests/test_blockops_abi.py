"""The operators of residual blocks and classifiers at the C boundary, without
a GPU: signatures of the binding against the header, refusals before any
device work, workspace sizes, the wrapper's and the model's own checks."""
import ctypes
import os
import re

import pytest
import torch

from paper_2607_17374_amd import _native as N
import paper_2607_17374_amd as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = ("taurus_linear_bytes", "taurus_linear", "taurus_linear_grad_bytes", "taurus_linear_grad",
         "taurus_residual_norm", "taurus_residual_norm_grad_bytes", "taurus_residual_norm_grad",
         "taurus_label_log_probs_bytes", "taurus_label_log_probs", "taurus_label_log_probs_grad")


def test_argument_types_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "taurus.h")).read(), flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "int": ctypes.c_int}
    for name in CALLS:
        m = re.search(r"(\w+)\s+%s\s*\(([^)]*)\)\s*;" % name, text)
        want = [ctypes.c_void_p if "*" in p else kinds[p.split()[0]] for p in m.group(2).split(",")]
        assert N.SIGNATURES[name][1] == want, name
        assert N.SIGNATURES[name][0] == kinds[m.group(1)], name


def test_assembly_leaves_m0_as_it_was():
    """m0 is reserved, so no clobber tells the compiler that assembly writes it:
    what writes it saves it first and puts it back last."""
    csrc, found = os.path.join(ROOT, "paper_2607_17374_amd", "csrc"), 0
    for name in sorted(os.listdir(csrc)):
        for block in re.findall(r"\basm\b[^(;]*\((.*?)\);", open(os.path.join(csrc, name)).read(), flags=re.S):
            lines = [x for s in re.findall(r'"([^"]*)"', block.split("\n        :")[0]) for x in s.split("\\n\\t") if x]
            if not any(re.match(r"\w+ m0,", x) for x in lines):
                continue
            found += 1
            saved = re.fullmatch(r"s_mov_b32 (%\d+), m0", lines[0])
            assert saved and lines[-1] == f"s_mov_b32 m0, {saved.group(1)}", (name, lines)
    assert found


P = 1 << 20  # a pointer no refused call follows


def _linear(**kw):
    a = dict(x=P, dt=N.BF16, m=16, k=8, xs=8, w=P, n=8, bias=None, res=None, rs=8, act=0, out=P, odt=N.F32, os=8,
             pre=None, ps=8, work=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return N.lib().taurus_linear(*a.values())


def _linear_grad(**kw):
    a = dict(grad=P, gs=8, x=P, xs=8, dt=N.BF16, m=16, k=8, n=8, w=P, pre=P, ps=8, act=N.ACT_SILU, dx=P, dxs=8, dw=P,
             wdt=N.F32, db=P, work=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return N.lib().taurus_linear_grad(*a.values())


def _resnorm(**kw):
    a = dict(x=P, xdt=N.BF16, xs=8, f=P, dt=N.BF16, fs=8, m=16, d=8, scale=1.0, gate=None, off=None, segs=0,
             post=N.NORM_RMS, pw=None, pb=None, pe=1e-5, pre=N.NORM_LAYER, qw=None, qb=None, qe=1e-5, y=P, ys=8, h=P,
             hs=8, stats=None, stream=None)
    a.update(kw)
    return N.lib().taurus_residual_norm(*a.values())


def _resnorm_grad(**kw):
    a = dict(gy=P, gys=8, gh=P, ghs=8, y=P, ydt=N.BF16, ys=8, f=P, dt=N.BF16, fs=8, m=16, d=8, scale=1.0, gate=None,
             off=None, segs=0, post=N.NORM_RMS, pw=None, pb=None, pre=N.NORM_LAYER, qw=None, stats=P, dx=P, dxs=8, df=P,
             dfs=8, dgate=None, dpw=None, dpb=None, dqw=None, dqb=None, work=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return N.lib().taurus_residual_norm_grad(*a.values())


def _labels(**kw):
    a = dict(x=P, dt=N.BF16, m=16, c=8, xs=8, labels=P, scale=1.0, top=2, logp=P, stats=P, entropy=P, tv=P, ti=P,
             work=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return N.lib().taurus_label_log_probs(*a.values())


def _labels_grad(**kw):
    a = dict(x=P, dt=N.BF16, m=16, c=8, xs=8, labels=P, scale=1.0, stats=P, entropy=P, g=P, h=P, dx=P, ds=8, stream=None)
    a.update(kw)
    return N.lib().taurus_label_log_probs_grad(*a.values())


BAD = [
    (_linear, dict(dt=7), "none of"), (_linear, dict(odt=7), "none of"), (_linear, dict(m=-1), "rows"),
    (_linear, dict(m=1 << 31), "rows"), (_linear, dict(k=0), "input width"), (_linear, dict(n=0), "output width"),
    (_linear, dict(k=(1 << 20) + 1), "input width"), (_linear, dict(n=(1 << 20) + 1), "output width"),
    (_linear, dict(act=5), "activation"), (_linear, dict(act=-1), "activation"), (_linear, dict(w=None), "weight is null"),
    (_linear, dict(x=None), "x is null"), (_linear, dict(out=None), "out is null"), (_linear, dict(xs=7), "apart"),
    (_linear, dict(os=7), "apart"), (_linear, dict(res=P, rs=7), "apart"), (_linear, dict(pre=P, ps=7), "apart"),
    (_linear, dict(bias=P + 2), "bias is not aligned"), (_linear, dict(x=P + 1), "x is not aligned"),
    (_linear, dict(res=P + 2), "residual is not aligned"), (_linear, dict(pre=P + 1), "pre is not aligned"),
    (_linear, dict(m=100, k=4096, xs=4096, bytes=16), "workspace has 16"), (_linear, dict(m=100, k=4096, xs=4096, work=None), "workspace is null"),
    (_linear, dict(m=100, k=4096, xs=4096, work=P + 4), "16-byte aligned"),
    (_linear_grad, dict(wdt=5), "none of"), (_linear_grad, dict(gs=7), "apart"), (_linear_grad, dict(xs=7), "apart"),
    (_linear_grad, dict(dxs=7), "apart"), (_linear_grad, dict(w=None), "weight is null"),
    (_linear_grad, dict(x=None), "x is null"), (_linear_grad, dict(pre=None), "pre is null"),
    (_linear_grad, dict(ps=7), "apart"), (_linear_grad, dict(bytes=1), "workspace has 1"),
    (_linear_grad, dict(work=None), "workspace is null"), (_linear_grad, dict(dw=P + 2), "dweight is not"),
    (_linear_grad, dict(db=P + 2), "dbias is not"), (_linear_grad, dict(act=9), "activation"),
    (_resnorm, dict(dt=3), "none of"), (_resnorm, dict(xdt=3), "none of"), (_resnorm, dict(xdt=N.F16), "fp32"),
    (_resnorm, dict(dt=N.F32, xdt=N.BF16), "fp32"), (_resnorm, dict(d=0), "channels"),
    (_resnorm, dict(d=8193, xs=8193, fs=8193, ys=8193, hs=8193), "channels"), (_resnorm, dict(m=-1), "rows"),
    (_resnorm, dict(post=3), "norm 3"), (_resnorm, dict(pre=-1), "norm -1"), (_resnorm, dict(pe=-1.0), "eps"),
    (_resnorm, dict(qe=float("nan")), "eps"), (_resnorm, dict(x=None), "x is null"), (_resnorm, dict(f=None), "f is null"),
    (_resnorm, dict(y=None), "y is null"), (_resnorm, dict(h=None), "h is null"), (_resnorm, dict(xs=7), "apart"),
    (_resnorm, dict(fs=7), "apart"), (_resnorm, dict(ys=7), "apart"), (_resnorm, dict(hs=7), "apart"),
    (_resnorm, dict(gate=P + 2), "gate is not"), (_resnorm, dict(off=P + 4, segs=2), "off is not aligned"),
    (_resnorm, dict(off=P, segs=-1), "segments"), (_resnorm, dict(pw=P + 1), "not aligned"),
    (_resnorm, dict(qb=P + 1), "not aligned"), (_resnorm, dict(stats=P + 4), "stats is not aligned"),
    (_resnorm_grad, dict(gh=None), "grad_h is null"), (_resnorm_grad, dict(y=None), "y is null"),
    (_resnorm_grad, dict(f=None), "f is null"), (_resnorm_grad, dict(stats=None), "stats is null"),
    (_resnorm_grad, dict(gys=7), "apart"), (_resnorm_grad, dict(dxs=7), "apart"), (_resnorm_grad, dict(dfs=7), "apart"),
    (_resnorm_grad, dict(dgate=P), "gate that there is not"), (_resnorm_grad, dict(post=0, dpw=P), "there is not"),
    (_resnorm_grad, dict(pre=0, gh=None, dqb=P), "there is not"), (_resnorm_grad, dict(pre=0), "h, which there is not"),
    (_resnorm_grad, dict(bytes=8), "workspace has 8"), (_resnorm_grad, dict(work=None), "workspace is null"),
    (_resnorm_grad, dict(dpw=P + 2), "not aligned"), (_resnorm_grad, dict(ydt=N.F16), "fp32"),
    (_labels, dict(dt=3), "none of"), (_labels, dict(c=0), "classes"), (_labels, dict(c=(1 << 22) + 1), "classes"),
    (_labels, dict(m=-1), "rows"), (_labels, dict(scale=0.0), "scale"), (_labels, dict(scale=-1.0), "scale"),
    (_labels, dict(scale=float("inf")), "scale"), (_labels, dict(scale=float("nan")), "scale"),
    (_labels, dict(top=-1), "alternatives"), (_labels, dict(top=9), "alternatives"),
    (_labels, dict(c=100, xs=100, top=65), "alternatives"), (_labels, dict(labels=None), "labels is null"),
    (_labels, dict(tv=None), "top_logp is null"), (_labels, dict(ti=None), "top_ids is null"),
    (_labels, dict(x=None), "x is null"), (_labels, dict(xs=7), "apart"), (_labels, dict(stats=P + 2), "not aligned"),
    (_labels, dict(c=50_000, xs=50_000, bytes=8), "workspace has 8"),
    (_labels, dict(c=50_000, xs=50_000, work=None), "workspace is null"),
    (_labels_grad, dict(stats=None), "stats is null"), (_labels_grad, dict(g=None), "grad_logp is null"),
    (_labels_grad, dict(entropy=None), "entropy is null"), (_labels_grad, dict(dx=None), "dx is null"),
    (_labels_grad, dict(ds=7), "apart"), (_labels_grad, dict(scale=0.0), "scale"), (_labels_grad, dict(h=P + 1), "not aligned"),
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_refused_before_device_work(i):
    call, change, text = BAD[i]
    assert call(**change) == N.E_INVALID, change
    assert text in N.last_error(), N.last_error()


def test_nothing_to_do_is_ok_without_pointers():
    assert _linear(m=0, x=None, out=None, w=None, work=None) == N.OK
    assert _linear_grad(dx=None, dw=None, db=None, grad=None, x=None, work=None) == N.OK
    assert _resnorm(m=0, x=None, f=None, y=None, h=None) == N.OK
    assert _resnorm(off=P, segs=0) == N.OK
    assert _labels(m=0, x=None, labels=None, logp=None, work=None) == N.OK
    assert _labels_grad(m=0, x=None, dx=None, stats=None) == N.OK


def test_workspace_sizes():
    L = N.lib()
    assert L.taurus_linear_bytes(N.BF16, 1_000_000, 256, 256) == 0       # tiles fill the chip
    assert L.taurus_linear_bytes(N.BF16, 32, 1024, 1024) == 0            # few rows: one launch
    assert L.taurus_linear_bytes(N.BF16, 32, 4096, 1024) >= 2 * 32 * 1024 * 4
    assert L.taurus_linear_bytes(N.BF16, 65, 4096, 1024) >= 2 * 65 * 1024 * 4
    assert L.taurus_label_log_probs_bytes(N.BF16, 100_000, 1000, 5) == 0
    assert L.taurus_label_log_probs_bytes(N.BF16, 3, 100_000, 5) > 0
    # dz, where there is an activation
    assert (L.taurus_linear_grad_bytes(N.BF16, 100_000, 64, 64, N.ACT_SILU)
            >= L.taurus_linear_grad_bytes(N.BF16, 100_000, 64, 64, N.ACT_NONE) + 100_000 * 64 * 2)
    for bad in (L.taurus_linear_bytes(N.F32, -1, 4, 4), L.taurus_linear_bytes(5, 4, 4, 4), L.taurus_linear_grad_bytes(N.F32, 4, 0, 4, 0),
                L.taurus_linear_grad_bytes(N.F32, 4, 4, 4, 7), L.taurus_residual_norm_grad_bytes(N.F32, 4, 8193, 0, 0),
                L.taurus_residual_norm_grad_bytes(N.F32, 4, 8, -1, 1), L.taurus_label_log_probs_bytes(N.F32, 4, 4, 5)):
        assert bad == N.E_INVALID


@pytest.mark.parametrize("dtype,size", [(N.F32, 4), (N.BF16, 2)])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (5, 4096, 11008), (300, 64, 64), (100_000, 256, 256), (16_384, 4096, 4096),
                                   (30_000_000, 128, 47), (7, 1 << 20, 64), (7, 64, 1 << 20), (4096, 1 << 16, 1 << 16)])
def test_linear_workspace_is_bounded(dtype, size, m, k, n):
    """Parts' sums: a tile of 128 x 128 for each of 1,024 workgroups at most;
    the gradient's besides hold dz and a row of sums for every 32 rows or each
    of 2,048 workgroups of at least a tile's columns."""
    parts = 1024 * 128 * 128 * 4
    assert 0 <= N.lib().taurus_linear_bytes(dtype, m, k, n) <= parts + 256
    for act in (N.ACT_NONE, N.ACT_GELU):
        dz = 0 if act == N.ACT_NONE else m * (n + 7) * size
        sums = min(m // 32 + 1, 2048 * 256 // n + 1) * n * 4
        assert N.lib().taurus_linear_grad_bytes(dtype, m, k, n, act) <= parts + dz + sums + 2048 * 512 * 4 + 1024


@pytest.mark.parametrize("dtype,m,k,n", [
    (N.BF16, 40, 4096, 50), (N.BF16, 1_000_000, 64, 64), (N.BF16, 1_000_000, 1, 1), (N.F32, 1_000_000, 64, 64),
    (N.F16, 200_000, 1000, 47), (N.BF16, 16_384, 2048, 8191), (N.F32, 300_000, 256, 255), (N.BF16, 255, 8192, 8192),
    (N.F32, 700, 512, 512), (N.BF16, 700, 1024, 1024),
])
def test_no_workspace_for_large_tiles_that_sizes_rule_out(dtype, m, k, n):
    """Widths that are no whole 16-byte pieces, less than 256 a side or few
    multiply-adds leave only parts of the smaller tiles, of at least four stages
    each: as many sums of the product itself, not of tiles of 256 x 256."""
    size, stage = (4, 32) if dtype == N.F32 else (2, 64)

    def parts(rows, cols, depth):
        n = min(1024, -(-depth // stage) // 4)
        return n * rows * cols * 4 if n > 1 else 0

    assert N.lib().taurus_linear_bytes(dtype, m, k, n) <= parts(m, n, k) + 256
    sums = min(m // 32 + 1, 2048) * n * 4
    if m >= 256:  # a gradient of fewer rows can have a side that is taken
        assert N.lib().taurus_linear_grad_bytes(dtype, m, k, n, N.ACT_NONE) <= max(parts(m, k, n), parts(k, n, m)) + sums + 512


def test_label_kernels_are_those_that_rows_reach():
    """Every kernel of rows in registers is some number of classes', and every
    number has its own: vectors a row's type and width allow, sixteen values a
    lane, three vectors of fp32 where they hold the row."""
    reached = set()
    for dtype in (N.F32, N.BF16, N.F16):
        for c in range(1, 1025):
            e = 4 if dtype == N.F32 else 8
            while e > c:
                e //= 2
            vecs, p, lg = -(-c // e), 1, 0
            while p < 16 // e and vecs > p:
                p *= 2
            while vecs > p << lg:
                lg += 1
            if (e, p) == (4, 4) and vecs <= 3 << lg:
                p = 3
            reached.add((dtype, e, p, lg))
    names = re.findall(rb"k_labels_rowsILi(\d)ELi(\d)ELi(\d)ELi(\d)EEE", open(N.LIB_PATH, "rb").read())
    assert {tuple(int(v) for v in n) for n in names} == reached


def test_refused_sizes_are_told_every_time():
    from paper_2607_17374_amd import blockops
    for _ in range(2):
        with pytest.raises(T.TaurusError, match="alternatives"):
            blockops._bytes("taurus_label_log_probs_bytes", N.F32, 4, 4, 5)
        N.lib().taurus_linear_bytes(N.F32, -1, 4, 4)  # another message in between


def test_wrapper_refuses_host_tensors():
    x, v, ids = torch.zeros(4, 8), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    w = torch.zeros(8, 8)
    for call in (lambda: T.linear(x, w), lambda: T.linear_grad(x, x, w), lambda: T.residual_norm(x, x),
                 lambda: T.residual_norm_grad(x, None, x, x, None), lambda: T.label_log_probs(x, ids),
                 lambda: T.label_log_probs_grad(x, ids, torch.zeros(4, 2), v)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="need names"):
        T.linear_grad(x, x, w, need=("dx",))
    with pytest.raises(ValueError, match="need names"):
        T.residual_norm_grad(x, x, x, x, None, need=("y",))
    with pytest.raises(ValueError, match="go together"):
        T.label_log_probs_grad(x, ids, torch.zeros(4, 2), None)
    with pytest.raises(ValueError, match="go together"):
        T.label_log_probs_grad(x, None, torch.zeros(4, 2), None, grad_entropy=v)


LAYER = dict(d_in=8, d_out=8)


@pytest.mark.parametrize("layers,head,text", [
    ([dict(LAYER, residual=dict(gates=1))], None, "residual does not know gates"),
    ([dict(LAYER, residual=dict(post=dict(act="relu")))], None, "post does not know act"),
    ([dict(LAYER, residual=dict(pre=dict(kind="group")))], None, "pre's kind"),
    ([dict(LAYER, residual={}, norm=dict(groups=2))], None, "a norm or a residual"),
    ([dict(d_in=8, d_out=4, residual={})], None, "8 to 4 values has no residual"),
    ([dict(LAYER, out_dtype=N.BF16), dict(LAYER, out_dtype=N.F16, residual={})], None, "the residual stream is"),
    ([dict(LAYER)], dict(labelz=1), "head does not know labelz"),
    ([dict(LAYER)], dict(linear=[dict(bias=1)]), "head's linear maps"),
    ([dict(LAYER)], dict(linear=[dict(weight=1, residual=2)]), "head's linear maps"),
    ([dict(LAYER)], dict(linear=[dict(weight=torch.zeros(9, 4))]), "takes no rows of 8 values"),
    ([dict(LAYER)], dict(linear=[dict(weight=torch.zeros(8, 4)), dict(weight=torch.zeros(5, 4))]), "takes no rows of 4 values"),
    ([dict(LAYER)], dict(labels=torch.zeros(5)), "5 labels for 4 vertices"),
])
def test_model_refuses_blocks_and_heads_that_do_not_fit(layers, head, text):
    x, off = torch.zeros(4, 8), torch.tensor([0, 4])
    with pytest.raises(ValueError, match=text):
        T.run_layers(4, off, x, x, layers, chunk=4, head=head)


V8, ELSEWHERE = torch.zeros(8), torch.zeros(8, device="meta")  # the graph is on the CPU


@pytest.mark.parametrize("block,text", [
    (dict(gate=torch.zeros(9)), "gate must be contiguous with shape"), (dict(gate=V8.double()), "gate must be torch.float32"),
    (dict(gate=ELSEWHERE), "gate must be on cpu"), (dict(gate=torch.zeros(16)[::2]), "gate must be contiguous"),
    (dict(gate=V8, off=torch.tensor([0, 4])), "gate must be contiguous with shape"),
    (dict(gate=torch.zeros(2, 8), off=torch.tensor([0, 4])), "gate must be contiguous with shape"),
    (dict(off=torch.tensor([0, 4], dtype=torch.int32)), "off must be torch.int64"),
    (dict(off=torch.tensor([[0, 4]])), "off must be contiguous"), (dict(off=torch.zeros(0, dtype=torch.int64)), "^off must be"),
    (dict(off=torch.zeros(2, dtype=torch.int64, device="meta")), "off must be on cpu"),
    (dict(post=dict(weight=torch.zeros(7))), "post's weight must be contiguous"),
    (dict(post=dict(bias=V8.to(torch.bfloat16))), "post's bias must be torch.float32"),
    (dict(pre=dict(weight=ELSEWHERE)), "pre's weight must be on cpu"), (dict(pre=dict(bias=torch.zeros(1, 8))), "pre's bias"),
    (dict(pre=dict(eps=-1.0)), "pre's eps"), (dict(post=dict(kind="rms", eps=float("nan"))), "post's eps"),
])
def test_model_refuses_a_blocks_arrays_before_any_layer(block, text):
    """In the second layer, so that the first would have run."""
    x, off = torch.zeros(4, 8), torch.tensor([0, 4])
    with pytest.raises(ValueError, match=text):
        T.run_layers(4, off, x, x, [dict(LAYER), dict(LAYER, residual=block)], chunk=4)


def test_model_refuses_blocks_of_too_many_channels():
    x, off, wide = torch.zeros(4, 8), torch.tensor([0, 4]), dict(d_in=8193, d_out=8193)
    with pytest.raises(ValueError, match="at most 8192 channels"):
        T.run_layers(4, off, x, x, [dict(wide), dict(wide, residual={})], chunk=4)
    assert _resnorm(d=N.RESIDUAL_MOST + 1, xs=1 << 14, fs=1 << 14, ys=1 << 14, hs=1 << 14) == N.E_INVALID


W84, HALF84 = torch.zeros(8, 4), torch.zeros(8, 4, dtype=torch.bfloat16)


@pytest.mark.parametrize("head,text", [
    (dict(linear=[dict(weight=HALF84)]), "weight of a head's linear map must be torch.float32"),
    (dict(linear=[dict(weight=W84), dict(weight=HALF84[:4])]), "weight of a head's linear map must be torch.float32"),
    (dict(linear=[dict(weight=torch.zeros(4, 8).t())]), "weight of a head's linear map must be contiguous"),
    (dict(linear=[dict(weight=torch.zeros(8, 4, device="meta"))]), "weight of a head's linear map must be on cpu"),
    (dict(linear=[dict(weight=W84, bias=torch.zeros(5))]), "bias of a head's linear map must be contiguous"),
    (dict(linear=[dict(weight=W84, bias=HALF84[0])]), "bias of a head's linear map must be torch.float32"),
    (dict(linear=[dict(weight=W84, act="tanh")]), "act must be one of"),
    (dict(labels=torch.zeros(4, dtype=torch.int64)), "labels must be torch.int32"),
    (dict(labels=torch.zeros(4, dtype=torch.int32, device="meta")), "labels must be on cpu"),
    (dict(labels=torch.zeros(2, 2, dtype=torch.int32)), "labels must be contiguous"),
    (dict(top=9), r"top 9 is not in \[0, 8\]"), (dict(top=-1), "top -1"), (dict(linear=[dict(weight=W84)], top=5), r"\[0, 4\]"),
    (dict(linear=[dict(weight=torch.zeros(8, 99))], top=65), r"\[0, 64\]"),
    (dict(linear=[dict(weight=torch.zeros(8, 0))]), "1 to 4194304 classes, not 0"),
    (dict(scale=0.0), "scale 0.0"), (dict(scale=float("nan")), "scale nan"), (dict(scale=float("inf")), "scale inf"),
])
def test_model_refuses_a_head_before_any_layer(head, text):
    x, off = torch.zeros(4, 8), torch.tensor([0, 4])
    with pytest.raises(ValueError, match=text):
        T.run_layers(4, off, x, x, [dict(LAYER)], chunk=4, head=head)


@pytest.mark.parametrize("layers,dtype", [
    ([dict(LAYER, out_dtype=N.BF16)], torch.bfloat16), ([dict(LAYER)], torch.float32), ([], torch.float16),
    ([dict(LAYER, out_dtype=N.F16, residual={})], torch.float16),
    ([dict(LAYER), dict(LAYER, out_dtype=N.BF16, residual={})], torch.float32),  # y: the stream's type
    ([dict(LAYER), dict(LAYER, out_dtype=N.BF16, residual=dict(pre=dict(kind="rms")))], torch.bfloat16),
    ([dict(LAYER), dict(LAYER, out_dtype=N.BF16, residual=dict(pre={})), dict(LAYER, out_dtype=N.F16, in_dtype=N.BF16)], torch.float16),
])
def test_model_knows_the_type_that_the_head_takes(layers, dtype):
    """Maps of the rows' type pass the checks (and end at the graph, which is no
    device tensor here); those of another type are refused."""
    x, off = torch.zeros(4, 8, dtype=torch.float16), torch.tensor([0, 4])
    for other in (torch.float32, torch.bfloat16, torch.float16):
        text = "row_off must be a device tensor" if other == dtype else "weight of a head's linear map must be"
        with pytest.raises(ValueError, match=text):
            T.run_layers(4, off, x, x, layers, chunk=4, head=dict(linear=[dict(weight=torch.zeros(8, 4, dtype=other))], top=4))


def _meta(dtype=torch.float32, d=8):
    return torch.zeros(4, d, dtype=dtype, device="meta")


HOST, BLOCK, SHARED = "where the graph is", dict(LAYER, residual={}), torch.zeros(4, 8)


@pytest.mark.parametrize("x,layers,outs,head,text", [
    (_meta(), [BLOCK], None, None, "x must be on cpu, " + HOST),
    (SHARED, [dict(LAYER), BLOCK], [_meta(), None], None, r"outs\[0\] must be on cpu, " + HOST),
    (SHARED, [dict(LAYER), BLOCK], [None, _meta()], None, r"outs\[1\] must be on cpu, " + HOST),
    (SHARED, [dict(LAYER)], [_meta()], {}, r"outs\[0\] must be on cpu, " + HOST),
    (_meta(), [dict(LAYER)], None, {}, r"outs\[0\] must be on cpu, " + HOST),  # made where x is
    (_meta(), [], None, {}, "x must be on cpu, " + HOST),
    (SHARED, [dict(LAYER), BLOCK], [None, torch.zeros(4, 8, dtype=torch.float16)], None, r"outs\[1\] must hold the residual stream"),
    (SHARED, [dict(LAYER), BLOCK], [None, torch.zeros(5, 8)], None, r"outs\[1\] must hold the residual stream"),
    (SHARED, [dict(LAYER), dict(BLOCK, out_dtype=N.BF16)], [None, torch.zeros(4, 8, dtype=torch.bfloat16)], None,
     r"outs\[1\] must hold the residual stream, torch.float32"),
    (SHARED, [BLOCK], [SHARED], None, r"outs\[0\] overlaps"),
    (SHARED, [dict(LAYER), BLOCK], [torch.zeros(4, 8)] * 2, None, r"outs\[1\] overlaps"),
    # a plain layer's rows may be anywhere, and a block's given outputs be the stream
    (_meta(), [dict(LAYER)], [_meta()], None, "row_off must be a device tensor"),
    (_meta(), [dict(LAYER), BLOCK], [torch.zeros(4, 8), torch.zeros(4, 8)], {}, "row_off must be a device tensor"),
    (SHARED, [BLOCK, dict(BLOCK, out_dtype=N.BF16)], [torch.zeros(4, 8), torch.zeros(4, 8)], {}, "row_off must be a device tensor"),
])
def test_model_refuses_rows_that_lie_elsewhere_before_any_layer(x, layers, outs, head, text):
    with pytest.raises(ValueError, match=text):
        T.run_layers(4, torch.tensor([0, 4]), SHARED, x, layers, chunk=4, outs=outs, head=head)


def test_model_takes_the_table_of_an_encoder_as_output():
    """The encoder's rows are new: a block may write over the table they came
    from (the call ends at the lookup, which the table's place is refused by)."""
    x, off = torch.zeros(4, 8), torch.tensor([0, 4])
    with pytest.raises(ValueError, match="table must be a device tensor"):
        T.run_layers(4, off, x, x, [BLOCK], chunk=4, outs=[x], encoder=dict(ids=torch.zeros(4, dtype=torch.int32)))


class _FakeRun:
    """run_layers' parts as a log of what they are asked, without a device."""

    def __init__(self, monkeypatch):
        self.log = log = []

        class FakeLayer:
            def __init__(self, n, row_off, col_dst, out, **kw):
                self.out = out

            def push_all(self, h):
                log.append(("push", h))

            def finalize(self):
                return {}

            def destroy(self):
                pass

        class FakePlan:
            def __init__(self, *a, **kw):
                pass

            def destroy(self):
                pass

        def residual(x, f, out=None, stream=None, pre=None, **kw):
            log.append(("block", x))
            return out, torch.ones_like(f) if pre else None

        def answer(h, head, stream):
            log.append(("answer", h))
            return T.LabelLogProbs(None, None, None, None, None)
        monkeypatch.setattr(T.api, "Layer", FakeLayer)
        monkeypatch.setattr(T.api, "Plan", FakePlan)
        monkeypatch.setattr(T.api, "residual_norm", residual)
        monkeypatch.setattr(T.api, "_answer", answer)

    def synchronize(self):  # the run's stream
        self.log.append(("wait", None))

    def __call__(self, layers, **kw):
        self.x = torch.zeros(6, 8)
        return T.run_layers(4, None, None, self.x, layers, chunk=4, stream=self, **kw)


def test_model_carries_the_residual_stream(monkeypatch):
    """A block's stream is what the block before put out, the next layer's
    input its pre; the stream keeps fp32 beside layers of 16 bits."""
    run = _FakeRun(monkeypatch)
    block = dict(LAYER, out_dtype=N.BF16, residual=dict(pre=dict(kind="rms")))
    outs, _ = run([block, block, dict(block, residual={})], head=dict(top=0))
    kinds, args = zip(*run.log)
    assert kinds == ("push", "block") * 3 + ("answer", "wait")
    assert args[1].data_ptr() == run.x.data_ptr() and args[1].shape == (4, 8)  # the first layer's input, n rows
    assert args[2].dtype == torch.bfloat16 and (args[2] == 1).all()             # pre of the first block
    assert args[3] is outs[0] and args[5] is outs[1] and args[6].data_ptr() == outs[2].data_ptr()
    assert all(o.dtype == torch.float32 for o in outs[:3]) and isinstance(outs[3], T.LabelLogProbs)
    run.log.clear()
    run([LAYER])
    assert [k for k, _ in run.log] == ["push"]


def test_model_puts_a_blocks_output_where_its_rows_are(monkeypatch):
    """Behind a plain layer that streams x from elsewhere into a given output."""
    run = _FakeRun(monkeypatch)
    given = torch.zeros(4, 8)
    outs, _ = T.run_layers(4, None, None, _meta(), [LAYER, BLOCK], chunk=4, stream=run, outs=[given, None], head=dict(top=0))
    assert outs[0] is given and outs[1].device == given.device
    assert [k for k, _ in run.log] == ["push", "push", "block", "answer", "wait"]
