"""deco_layernorm, deco_layernorm_grad, deco_pack8 and deco_unpack8 against their definitions in 64 bits.

Tolerances.  eps = 2^-24 (fp32 rounding), d = u - mean.  A sum over a row passes at most 32 additions in a thread (rows of more
than 32768 columns: cols / 1024), 5 in a warp and 32 over warps: `depth` = 80 + cols / 1024 roundings, each of at most
eps times the sum of magnitudes.

  mean     4 eps |mean| + depth eps mean|d|
  rstd     relative: every d^2 carries 3 eps, the sum depth, the root halves it, root and quotient add 2: (depth + 10) eps
  y        |w| rstd (tol of mean + eps |d|) + |xhat w| (tol of rstd + 3 eps) + eps |y|, and half a unit of the type
  dx       xhat carries 2 eps, g one, c1 = mean g: depth eps mean|g|, c2 = mean(g xhat): (depth + 4) eps mean|g xhat|;
           dx: rstd (tol c1 + |xhat| tol c2 + 6 eps (|g| + |c1| + |xhat c2|)) + eps |dx|, and half a unit of the type
  dweight  a thread adds up rows / 148 rows at most, then up to 16 groups, 10 parts a warp and 5 steps of a tree: (rows / 148 + 64) eps
           sum |dy xhat|; dbias likewise of sum |dy|; and half a unit of the gradients' type

Checkpoints are compared bit by bit.
"""
import math

import pytest
import torch

from paper_2507_17346_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: EPS, torch.bfloat16: 2.0 ** -8}
NORM_EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    torch.cuda.set_device(0)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_of(rows, cols, dtype, seed, pad=0, lead=0, scale=1.0, offset=0.0):
    """[rows, cols] view with `pad` entries between rows and `lead` entries before the first."""
    stride = cols + pad
    buf = torch.full((lead + rows * stride + 64,), 1e4, device="cuda", dtype=DT[dtype])
    view = buf[lead:lead + rows * stride].view(rows, stride)[:, :cols]
    view.copy_((scale * torch.randn(rows, cols, generator=gen(seed), device="cuda") + offset).to(DT[dtype]))
    return view


def depth(cols):
    return 80 + cols / 1024


def near(got, want, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - want).abs() / tol.clamp_min(1e-300)
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g of the tolerance" % (what, worst)


def reference_norm(u, w, b):
    """y, mean, rstd and their tolerances, from u in its own type."""
    x = u.double()
    cols = x.shape[1]
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + NORM_EPS).rsqrt()
    w = torch.ones(cols, device="cuda", dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(cols, device="cuda", dtype=torch.float64) if b is None else b.double()
    y = d * rstd * w + b
    tm = 4 * EPS * mean.abs() + depth(cols) * EPS * d.abs().mean(1, keepdim=True) + 1e-40
    tr = (depth(cols) + 10) * EPS
    ty = w.abs() * rstd * (tm + EPS * d.abs()) + (d * rstd * w).abs() * (tr + 3 * EPS) + EPS * y.abs()
    ty = ty + HALF[u.dtype] * (y.abs() + ty) + 1e-40
    return y, mean.squeeze(1), rstd.squeeze(1), ty, tm.squeeze(1), tr * rstd.squeeze(1)


def run_norm(x, w, b, add=None, total=None, keep=False, y=None, stream=None):
    rows, cols = x.shape
    y = torch.full_like(x, 77.0) if y is None else y
    mean, rstd = torch.full((rows,), 77.0, device="cuda"), torch.full((rows,), 77.0, device="cuda")
    packed = B.packed8_empty(rows, cols) if keep else None
    if keep:
        packed[0].fill_(99)
        packed[1].fill_(99)
    B.deco_layernorm(x, w, b, y, mean=mean, rstd=rstd, eps=NORM_EPS, add=add, total=total, packed=packed, stream=stream)
    return y, mean, rstd, packed


def check_norm(u, w, b, y, mean, rstd):
    ry, rm, rr, ty, tm, tr = reference_norm(u, w, b)
    near(mean, rm, tm, "mean")
    near(rstd, rr, tr, "rstd")
    near(y, ry, ty, "y")


def reference_pack(x):
    """Codes and exponent bytes from the definition, in 64 bits."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    v = torch.zeros(rows, blocks * 32, dtype=torch.float64, device="cuda")
    v[:, :cols] = x.double()
    v = v.view(rows, blocks, 32)
    bad = ~torch.isfinite(v).all(2)
    v = torch.where(bad[:, :, None], torch.zeros_like(v), v)
    top = v.abs().amax(2)
    # the smallest e with top < 127.5 2^e (for 0 the smallest there is)
    e = torch.where(top > 0, torch.frexp(top / 127.5).exponent.long(), -126).clamp_min(-126)
    step = ((e + 1023) << 52).view(torch.float64)
    most = torch.where(e == 122, 63.0, 127.0)[:, :, None]           # 64 * 2^122 is no fp32 number
    q = torch.round(v / step[:, :, None]).clamp(-most, most)
    b = torch.where(bad, torch.full_like(e, 255), e + 127)
    return q.to(torch.int8).view(rows, -1), b.to(torch.uint8)


def values(packed, cols):
    codes, exps = packed
    step = ((exps.long() - 127 + 1023) << 52).view(torch.float64)
    return (codes.double() * step.repeat_interleave(32, 1))[:, :cols]


SHAPES = [(1, 1), (3, 2), (1, 768), (7, 31), (5, 32), (5, 33), (300, 100), (2, 1000), (9, 1024), (4, 1025), (3, 2048),
          (17, 4104), (2, 8192), (2, 8193), (2, 30001), (1, 32768), (2, 32769), (1, 70000), (2500, 64)]


# ------------------------------------------------------------------------------- forward

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(rows, cols, dtype):
    w = 1 + 0.3 * torch.randn(cols, generator=gen(1), device="cuda")
    b = torch.randn(cols, generator=gen(2), device="cuda")
    for pad, lead in ((0, 0), (3, 1), (8, 8)):
        x = rows_of(rows, cols, dtype, 3, pad, lead, 2.0, 0.5)
        y, mean, rstd, _ = run_norm(x, w, b)
        check_norm(x, w, b, y, mean, rstd)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (6, 96), (33, 100), (5, 2048), (3, 8197), (2, 40000)])
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_residual_and_checkpoint(rows, cols, dtype, pad, lead):
    x = rows_of(rows, cols, dtype, 4, pad, lead, 2.0)
    add = rows_of(rows, cols, dtype, 5, pad, lead, 3.0, -1.0)
    want = (x.float() + add.float()).to(x.dtype)
    total = rows_of(rows, cols, dtype, 6, pad, lead)
    y, mean, rstd, packed = run_norm(x, None, None, add, total, keep=True)
    assert torch.equal(total, want)
    check_norm(want, None, None, y, mean, rstd)
    q, e = reference_pack(want)
    assert torch.equal(packed[0], q) and torch.equal(packed[1], e)
    y2, _, _, _ = run_norm(x, None, None, add)                     # the sum need not be stored
    assert torch.equal(y2, y)
    y3, _, _, packed = run_norm(x, None, None, keep=True)
    check_norm(x, None, None, y3, *run_norm(x, None, None)[1:3])
    q, e = reference_pack(x)
    assert torch.equal(packed[0], q) and torch.equal(packed[1], e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [768, 1001, 40000])
def test_norm_in_place_and_over_the_residual(dtype, cols):
    x, add = rows_of(5, cols, dtype, 7), rows_of(5, cols, dtype, 8)
    want, _, _, _ = run_norm(x, None, None, add)
    total = (x.float() + add.float()).to(x.dtype)
    a, b = x.clone(), add.clone()
    run_norm(a, None, None, b, total=b, y=a)
    assert torch.equal(a, want) and torch.equal(b, total)


def test_norm_of_unusual_rows():
    """A common offset of 10^4, a constant row, tiny and large entries, a NaN, an infinity: only its own row is touched."""
    cols = 1000
    for c in (cols, 1024):
        x = torch.randn(7, c, generator=gen(9), device="cuda")
        x[0] += 1e4
        x[1] = 3.25
        x[2] *= 1e-20
        x[3] *= 1e15
        y, mean, rstd, _ = run_norm(x, None, None)
        check_norm(x, None, None, y, mean, rstd)
        assert (y[1] == 0).all()
        clean = y.clone()
        x[5, 17] = math.nan
        x[6, 0] = -math.inf
        y, mean, rstd, _ = run_norm(x, None, None)
        assert torch.equal(y[:5], clean[:5])
        assert y[5:].isnan().all() and rstd[5:].isnan().all()


# ------------------------------------------------------------------------------ checkpoints

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_pack_and_unpack(rows, cols, dtype):
    for pad, lead in ((0, 0), (3, 1), (8, 8)):
        x = rows_of(rows, cols, dtype, 10, pad, lead)
        x *= torch.exp(3 * torch.randn(rows, 1, generator=gen(11), device="cuda")).to(x.dtype)
        packed = B.packed8_empty(rows, cols)
        packed[0].fill_(99)
        B.deco_pack8(x, packed)
        q, e = reference_pack(x)
        assert torch.equal(packed[0], q) and torch.equal(packed[1], e)
        want = values(packed, cols)
        for out in ("f32", "bf16"):
            y = rows_of(rows, cols, out, 12, pad, lead)
            B.deco_unpack8(packed, y)
            assert torch.equal(y.double(), want)
        # at most half a step; a step is at most 2^-6 of the block's largest magnitude
        top = x.double().abs().amax()
        assert (want - x.double()).abs().max() <= top * 2.0 ** -7


@pytest.mark.parametrize("cols", [64, 61])
def test_pack_of_unusual_blocks(cols):
    big = torch.finfo(torch.float32).max
    x = torch.zeros(12, cols, device="cuda")
    x[0, :3] = torch.tensor([127.5, 1.5, 2.5])
    x[1, :3] = torch.tensor([127.49999, 0.5, 1.5])
    x[2, :2] = torch.tensor([-127.5 * 2.0 ** 60, 2.0 ** 59])
    x[3] = 1e-40
    x[4, :2] = torch.tensor([big, -big / 3])
    x[5] = -0.0
    x[6, 3], x[6, 4] = math.nan, 1.0
    x[7, 40] = math.inf
    x[8, 40] = -math.inf
    x[9, :2] = torch.tensor([2.0 ** -126, 2.0 ** -140])
    x[10] = torch.linspace(-1, 1, cols)
    x[11, :2] = torch.tensor([2.0 ** -120, 1.9921875 * 2.0 ** -121])
    packed = B.packed8_empty(12, cols)
    B.deco_pack8(x, packed)
    q, e = reference_pack(x)
    assert torch.equal(packed[0], q) and torch.equal(packed[1], e)
    for dtype in DT.values():
        y = torch.empty(12, cols, device="cuda", dtype=dtype)
        B.deco_unpack8(packed, y)
        bad = (e == 255).repeat_interleave(32, 1)[:, :cols]
        assert y[bad].isnan().all() and bad.sum() == 2 * (cols - 32) + 32
        assert torch.equal(y[~bad].double(), values(packed, cols)[~bad])
    once = B.packed8_empty(12, cols)                               # what was taken back gives the same again
    y = torch.empty(12, cols, device="cuda")
    B.deco_unpack8(packed, y)
    B.deco_pack8(y, once)
    z = torch.empty(12, cols, device="cuda")
    B.deco_unpack8(once, z)
    assert torch.equal(y.nan_to_num(5.0), z.nan_to_num(5.0))


# ------------------------------------------------------------------------------- gradient

def reference_grad(x, mean, rstd, w, dy, add):
    x, g0 = x.double(), dy.double()
    rows, cols = x.shape
    m, r = mean.double()[:, None], rstd.double()[:, None]
    w = torch.ones(cols, device="cuda", dtype=torch.float64) if w is None else w.double()
    h = (x - m) * r
    g = g0 * w
    c1, c2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = r * (g - c1 - h * c2)
    t1 = depth(cols) * EPS * g.abs().mean(1, keepdim=True)
    t2 = (depth(cols) + 4) * EPS * (g * h).abs().mean(1, keepdim=True)
    tol = r * (t1 + h.abs() * t2 + 6 * EPS * (g.abs() + c1.abs() + (h * c2).abs())) + EPS * dx.abs()
    if add is not None:
        dx = dx + add.double()
        tol = tol + EPS * dx.abs()
    tol = tol + HALF[dy.dtype] * (dx.abs() + tol) + 1e-40
    dep = (rows / 148 + 64) * EPS
    return dx, tol, (g0 * h).sum(0), dep * (g0 * h).abs().sum(0) + 1e-40, g0.sum(0), dep * g0.abs().sum(0) + 1e-40


def check_grad(x, mean, rstd, w, dy, add, dx, dw, db, old=0.0):
    rdx, tdx, rdw, tdw, rdb, tdb = reference_grad(x, mean, rstd, w, dy, add)
    near(dx, rdx, tdx, "dx")
    for got, want, tol, what in ((dw, rdw, tdw, "dweight"), (db, rdb, tdb, "dbias")):
        if got is not None:
            want = want + old
            near(got, want, tol + HALF[got.dtype] * (want.abs() + tol) + EPS * want.abs(), what)


def stats(x):
    d = x.double()
    return d.mean(1).float(), (d.var(1, correction=0) + NORM_EPS).rsqrt().float()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_grad(rows, cols, dtype):
    w = 1 + 0.3 * torch.randn(cols, generator=gen(20), device="cuda")
    for pad, lead in ((0, 0), (3, 1), (8, 8)):
        x = rows_of(rows, cols, dtype, 21, pad, lead, 2.0, 0.5)
        dy = rows_of(rows, cols, dtype, 22, pad, lead, 1e-2)
        mean, rstd = stats(x)
        dx = rows_of(rows, cols, dtype, 23, pad, lead)
        dw, db = torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
        B.deco_layernorm_grad(x, mean, rstd, w, dy, dx, dweight=dw, dbias=db)
        check_grad(x, mean, rstd, w, dy, None, dx, dw, db)


@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (40, 96), (33, 100), (1000, 776), (5, 2048), (3, 8197), (7, 40000)])
def test_grad_from_the_checkpoint_with_residual_and_accumulation(rows, cols, dtype, gtype):
    x = rows_of(rows, cols, dtype, 24, scale=2.0)
    mean, rstd = stats(x)
    packed = B.packed8_empty(rows, cols)
    B.deco_pack8(x, packed)
    dy, add = rows_of(rows, cols, dtype, 25, scale=1e-2), rows_of(rows, cols, dtype, 26, scale=1e-2)
    dx = torch.full_like(dy, 7.0)
    dw = torch.full((cols,), 0.5, device="cuda", dtype=DT[gtype])
    db = torch.full((cols,), 0.5, device="cuda", dtype=DT[gtype])
    B.deco_layernorm_grad(packed, mean, rstd, None, dy, dx, dweight=dw, dbias=db, add=add, accumulate=True)
    check_grad(values(packed, cols), mean, rstd, None, dy, add, dx, dw, db, old=0.5)
    again = torch.full_like(dx, 7.0)
    B.deco_layernorm_grad(packed, mean, rstd, None, dy, again, add=add)             # no sums wanted
    assert torch.equal(again, dx)
    one = torch.full((cols,), 3.0, device="cuda", dtype=DT[gtype])                   # one of the two, in place of dy
    over = dy.clone()
    B.deco_layernorm_grad(packed, mean, rstd, None, over, over, dbias=one, add=add)
    assert torch.equal(over, dx)
    check_grad(values(packed, cols), mean, rstd, None, dy, add, dx, None, one)


def test_grad_against_differences():
    """Central differences of a weighted sum of outputs, through the forward pass's own definition in 64 bits."""
    rows, cols = 3, 40
    x, w, b = (torch.randn(*s, generator=gen(27 + i), device="cuda") for i, s in enumerate([(rows, cols), (cols,), (cols,)]))
    dy = torch.randn(rows, cols, generator=gen(30), device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = torch.empty_like(x)
    B.deco_layernorm(x, w, b, y, mean=mean, rstd=rstd, eps=NORM_EPS)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.deco_layernorm_grad(x, mean, rstd, w, dy, dx, dweight=dw, dbias=db)

    def f(x, w, b):
        d = x - x.mean(1, keepdim=True)
        return (dy.double() * (d * (d.square().mean(1, keepdim=True) + NORM_EPS).rsqrt() * w + b)).sum()
    args = [t.double() for t in (x, w, b)]
    # step 1e-4: the third derivative's part is about 1e-8, rounding of the sums 1e-14 / 1e-4; both below 1e-5
    for which, got in ((0, dx), (1, dw), (2, db)):
        for i in (0, 7, got.numel() - 1):
            up, down = [t.clone() for t in args], [t.clone() for t in args]
            up[which].view(-1)[i] += 1e-4
            down[which].view(-1)[i] -= 1e-4
            diff = ((f(*up) - f(*down)) / 2e-4).item()
            assert abs(diff - got.view(-1)[i].item()) < 1e-5 * (1 + abs(diff))


def test_grad_of_no_rows():
    x = torch.empty(0, 100, device="cuda")
    e = torch.empty(0, device="cuda")
    dw, db = torch.full((100,), 5.0, device="cuda"), torch.full((100,), 5.0, device="cuda", )
    B.deco_layernorm_grad(x, e, e, None, x, x, dweight=dw, dbias=db, accumulate=True)
    assert (dw == 5).all() and (db == 5).all()
    B.deco_layernorm_grad(x, e, e, None, x, x, dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    B.deco_layernorm(x, None, None, x)
    B.deco_pack8(x, B.packed8_empty(0, 100))
    B.deco_unpack8(B.packed8_empty(0, 100), x)


def test_grad_touches_only_rows_with_a_nan():
    x = rows_of(50, 768, "f32", 31)
    dy = rows_of(50, 768, "f32", 32)
    mean, rstd = stats(x)
    clean, dx = torch.empty_like(x), torch.empty_like(x)
    B.deco_layernorm_grad(x, mean, rstd, None, dy, clean)
    dy[20, 3] = math.nan
    dw, db = torch.empty(768, device="cuda"), torch.empty(768, device="cuda")
    B.deco_layernorm_grad(x, mean, rstd, None, dy, dx, dweight=dw, dbias=db)
    assert dx[20].isnan().all() and dw[3].isnan() and db[3].isnan()
    keep = torch.arange(50, device="cuda") != 20
    assert torch.equal(dx[keep], clean[keep])
    rest = torch.arange(768, device="cuda") != 3
    assert torch.isfinite(dw[rest]).all() and torch.isfinite(db[rest]).all()


def test_same_bits_every_time():
    x, dy = rows_of(3000, 1000, "bf16", 33), rows_of(3000, 1000, "bf16", 34)
    mean, rstd = stats(x)
    first = None
    for _ in range(5):
        dx, dw, db = torch.empty_like(x), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
        room = torch.randint(0, 255, (B.deco_layernorm_grad_workspace(3000, 1000),), dtype=torch.uint8, device="cuda")
        B.deco_layernorm_grad(x, mean, rstd, None, dy, dx, dweight=dw, dbias=db, workspace=room)
        now = (dx, dw, db)
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now


# ----------------------------------------------------------- streams, graphs, far offsets

def test_two_streams_at_once_and_a_graph():
    x = rows_of(4000, 768, "bf16", 35)
    dy = rows_of(4000, 768, "bf16", 36)
    mean, rstd = stats(x)
    want = torch.empty(768, device="cuda"), torch.empty(768, device="cuda"), torch.empty_like(x)
    B.deco_layernorm_grad(x, mean, rstd, None, dy, want[2], dweight=want[0], dbias=want[1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for k in range(6):                                             # each call makes its own workspace, on its stream
        out = torch.empty(768, device="cuda"), torch.empty(768, device="cuda"), torch.empty_like(x)
        s = streams[k % 2]
        s.wait_stream(torch.cuda.current_stream())
        B.deco_layernorm_grad(x, mean, rstd, None, dy, out[2], dweight=out[0], dbias=out[1], stream=s)
        outs.append(out)
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    y = torch.empty_like(x)
    packed = B.packed8_empty(4000, 768)
    out = torch.zeros(768, device="cuda"), torch.zeros(768, device="cuda"), torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.deco_layernorm(x, None, None, y, mean=mean, rstd=rstd, eps=NORM_EPS, packed=packed)
        B.deco_layernorm_grad(x, mean, rstd, None, dy, out[2], dweight=out[0], dbias=out[1])
    x.copy_(rows_of(4000, 768, "bf16", 37))
    graph.replay()
    torch.cuda.synchronize()
    check_norm(x, None, None, y, mean, rstd)
    check_grad(x, mean, rstd, None, dy, None, out[2], out[0], out[1])
    assert torch.equal(packed[0], reference_pack(x)[0])


def test_rows_whose_offsets_pass_32_bits():
    rows, cols, stride = 3, 200, 2 ** 31 + 24
    buf = torch.zeros((rows - 1) * stride + cols, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (rows, cols), (stride, 1))
    x.copy_(rows_of(rows, cols, "bf16", 38))
    small = x.contiguous()
    want, mean, rstd, packed = run_norm(small, None, None, keep=True)
    again = B.packed8_empty(rows, cols)
    y = torch.empty_like(small)
    B.deco_layernorm(x, None, None, y, eps=NORM_EPS, packed=again)
    assert torch.equal(y, want) and torch.equal(again[0], packed[0])
    B.deco_layernorm(x, None, None, x, eps=NORM_EPS)
    assert torch.equal(x, want)
    B.deco_unpack8(packed, x)
    assert torch.equal(x.double(), values(packed, cols))
    dx = torch.empty_like(small)
    B.deco_layernorm_grad(packed, mean, rstd, None, want, dx)
    B.deco_layernorm_grad(packed, mean, rstd, None, want, x)
    assert torch.equal(x, dx)
    outside = torch.as_strided(buf, (rows - 1, stride - cols), (stride, 1), cols)
    for row in outside:
        assert not row.any()


# ------------------------------------------------------------------------------- refusals

def test_refusals():
    x = torch.randn(4, 100, device="cuda")
    y = torch.empty_like(x)
    v = torch.empty(4, device="cuda")
    packed = B.packed8_empty(4, 100)
    for bad in (x.half(), x.t(), x[0], x.double()):
        with pytest.raises(ValueError):
            B.deco_layernorm(bad, None, None, y)
        with pytest.raises(ValueError):
            B.deco_pack8(bad, packed)
    with pytest.raises(ValueError):
        B.deco_layernorm(x, torch.ones(99, device="cuda"), None, y)
    with pytest.raises(ValueError):
        B.deco_layernorm(x, None, None, y.bfloat16())
    with pytest.raises(ValueError):
        B.deco_layernorm(x, None, None, y, packed=B.packed8_empty(4, 96))
    with pytest.raises(ValueError):
        B.deco_layernorm_grad(x, v, v, None, x, y, dweight=torch.empty(100, device="cuda"),
                              dbias=torch.empty(100, device="cuda", dtype=torch.bfloat16))
    for eps in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(B.DecoError):
            B.deco_layernorm(x, None, None, y, eps=eps)
    with pytest.raises(B.DecoError):
        B.deco_layernorm(x, None, None, y, total=torch.empty_like(x))
    with pytest.raises(B.DecoError):
        B.deco_layernorm(x, None, None, y, add=x, total=y)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.DecoError) as e:
        B.deco_layernorm_grad(x, v, v, None, x, y, dweight=torch.empty(100, device="cuda"), workspace=small)
    assert e.value.status == B.DECO_ERR_CAPACITY
