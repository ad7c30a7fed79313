"""deco_weight_grad8 against its definition in 64 bits.

Tolerances.  eps = 2^-24, S = sum_t |dy_t x_t|.  Products are exact (bf16 times bf16 in fp32; fp32 dy is split into
three bf16 numbers without loss, into two with a loss of 2^-17 of each term).  The tensor cores cut sums off at 2^-23 of the sum at
each of the 32 additions (16 tokens each) of 512 tokens, and twice 32 more with small planes: 96 * 2 eps S.  Longer sums
are joined by rounded additions, rows / 512 of them: (rows / 512) eps S.  Where the result is bf16 nothing is joined: 2 eps S for each of
(rows / 16) * 2 additions; and half a unit, 2^-8 of the value.  So

  fp32 result    (192 + rows / 512) eps S
  bf16 result    (192 + rows / 4) eps S + 2^-17 S (fp32 dy) + 2^-8 |result|
"""
import math

import pytest
import torch

from paper_2507_17346_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


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


def randn(seed, *shape):
    return torch.randn(*shape, generator=gen(seed), device="cuda")


def checkpoint(rows, cols, seed, scale=1.0):
    packed = B.packed8_empty(rows, cols)
    B.deco_pack8(scale * randn(seed, rows, cols) * torch.exp(randn(seed + 1, rows, 1)), packed)
    return packed


def values(packed, cols):
    codes, exps = packed
    step = ((exps.long() - 127 + 1023) << 52).view(torch.float64)
    return (codes.double() * step.repeat_interleave(32, 1))[:, :cols]


def gradients(rows, out, dtype, seed, pad=0, lead=0):
    stride = out + pad
    buf = torch.full((lead + rows * stride + 64,), 1e4, device="cuda", dtype=DT[dtype])
    view = buf[lead:lead + rows * stride].view(rows, stride)[:, :out]
    view.copy_(1e-2 * randn(seed, rows, out))
    return view


def check(dy, packed, cols, dw, db, transposed, old=0.0):
    x, g = values(packed, cols), dy.double()
    rows = len(x)
    want, total = g.t() @ x, g.abs().t() @ x.abs()
    if transposed:
        want, total = want.t(), total.t()
    for got, want, total in ((dw, want, total), (db, g.sum(0), g.abs().sum(0))):
        if got is None:
            continue
        if got.dtype == torch.float32:
            tol = (192 + rows / 512) * EPS * total
        else:
            tol = (192 + rows / 4) * EPS * total + (2.0 ** -17 * total if dy.dtype == torch.float32 else 0)
        want = want + old
        tol = tol + EPS * want.abs() + 1e-40
        if got.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
        assert torch.isfinite(got).all()
        worst = ((got.double() - want).abs() / tol).max().item()
        assert worst <= 1.0, "%.3g of the tolerance" % worst


# (single CTAs, and in the last three pairs)
SHAPES = [(1, 1, 1), (2, 3, 5), (64, 128, 112), (63, 127, 113), (65, 129, 111), (100, 333, 129), (700, 64, 64), (513, 130, 600),
          (5000, 24, 40), (2048, 768, 768), (2000, 777, 1001), (4096, 256, 224), (1000, 2304, 700), (12000, 520, 330), (8192, 777, 1001), (4160, 1300, 1100), (16400, 530, 500)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,out,cols", SHAPES)
def test_weight_grad(rows, out, cols, dtype, gtype, transposed):
    packed = checkpoint(rows, cols, 1)
    shape = (cols, out) if transposed else (out, cols)
    for pad, lead, bias in ((0, 0, True), (3, 1, False), (8 - out % 8, 8, False)):
        dy = gradients(rows, out, dtype, 3, pad, lead)
        dw = torch.full(shape, 7.0, device="cuda", dtype=DT[gtype])
        db = torch.full((out,), 7.0, device="cuda", dtype=DT[gtype]) if bias else None
        B.deco_weight_grad8(dy, packed, dw, db=db, transposed=transposed)
        check(dy, packed, cols, dw, db, transposed)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,out,cols", [(70, 33, 50), (3000, 300, 500)])
def test_into_a_flat_vector_and_accumulation(rows, out, cols, gtype, transposed):
    """The matrix and the bias lie at odd places of a longer vector; what is around them stays."""
    flat = torch.full((7 + out * cols + 5 + out + 9,), 0.25, device="cuda", dtype=DT[gtype])
    shape = (cols, out) if transposed else (out, cols)
    dw = flat[7:7 + out * cols].view(shape)
    db = flat[7 + out * cols + 5:7 + out * cols + 5 + out]
    packed, dy = checkpoint(rows, cols, 5), gradients(rows, out, "bf16", 7)
    B.deco_weight_grad8(dy, packed, dw, db=db, transposed=transposed, accumulate=True)
    check(dy, packed, cols, dw, db, transposed, old=0.25)
    inside = torch.zeros_like(flat, dtype=torch.bool)
    inside[7:7 + out * cols] = True
    inside[7 + out * cols + 5:7 + out * cols + 5 + out] = True
    assert (flat[~inside] == 0.25).all()


@pytest.mark.parametrize("accumulate", [False, True])
def test_no_rows(accumulate):
    dw, db = torch.full((5, 9), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda")
    B.deco_weight_grad8(torch.empty(0, 5, device="cuda"), B.packed8_empty(0, 9), dw, db=db, accumulate=accumulate)
    assert (dw == (3.0 if accumulate else 0.0)).all() and (db == (3.0 if accumulate else 0.0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_no_numbers_stay_in_their_rows_and_columns(dtype):
    rows, out, cols = 300, 200, 150
    x = randn(8, rows, cols)
    x[17, 40] = math.nan                                           # its block of 32 columns
    packed = B.packed8_empty(rows, cols)
    B.deco_pack8(x, packed)
    dy = gradients(rows, out, dtype, 9)
    dy[33, 120] = math.nan
    dw, db = torch.empty(out, cols, device="cuda"), torch.empty(out, device="cuda")
    B.deco_weight_grad8(dy, packed, dw, db=db)
    bad = torch.zeros(out, cols, dtype=torch.bool, device="cuda")
    bad[120] = True
    bad[:, 32:64] = True
    assert dw[bad].isnan().all() and torch.isfinite(dw[~bad]).all()
    assert db[120].isnan() and torch.isfinite(db[:120]).all() and torch.isfinite(db[121:]).all()


def test_large_and_tiny_gradients():
    """fp32 gradients near the ends of the range are split without overflow."""
    rows, out, cols = 64, 32, 32
    packed = checkpoint(rows, cols, 10, 1e-3)
    dy = gradients(rows, out, "f32", 11)
    dy[:, 0] = 0.0
    dy[5, 0] = torch.finfo(torch.float32).max
    dy[:, 1] *= 1e-25
    dw, db = torch.empty(out, cols, device="cuda"), torch.empty(out, device="cuda")
    B.deco_weight_grad8(dy, packed, dw, db=db)
    check(dy, packed, cols, dw, db, False)


def test_same_bits_every_time_on_two_streams_and_in_a_graph():
    rows, out, cols = 4100, 700, 500
    packed, dy = checkpoint(rows, cols, 12), gradients(rows, out, "f32", 13)
    want, wb = torch.empty(out, cols, device="cuda"), torch.empty(out, device="cuda")
    B.deco_weight_grad8(dy, packed, want, db=wb)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for k in range(6):
        dw, db = torch.empty_like(want), torch.empty_like(wb)
        streams[k % 2].wait_stream(torch.cuda.current_stream())
        B.deco_weight_grad8(dy, packed, dw, db=db, stream=streams[k % 2])
        outs.append((dw, db))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) and torch.equal(b, wb) for a, b in outs)
    need = B.deco_weight_grad8_workspace(dy, cols)
    room = torch.randint(0, 255, (need,), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty_like(want), torch.empty_like(wb)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.deco_weight_grad8(dy, packed, dw, db=db, workspace=room)
    dy *= 2.0
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dw, 2 * want) and torch.equal(db, 2 * wb)


def test_refusals():
    dy, packed = torch.randn(64, 40, device="cuda"), B.packed8_empty(64, 48)
    dw = torch.empty(40, 48, device="cuda")
    for bad in (dy.half(), dy.t(), dy[0], dy.double()):
        with pytest.raises(ValueError):
            B.deco_weight_grad8(bad, packed, dw)
    with pytest.raises(ValueError):
        B.deco_weight_grad8(dy, packed, dw, transposed=True)
    with pytest.raises(ValueError):
        B.deco_weight_grad8(dy, packed, dw.half())
    with pytest.raises(ValueError):
        B.deco_weight_grad8(dy, packed, dw.t().contiguous().t())
    with pytest.raises(ValueError):
        B.deco_weight_grad8(dy, packed, dw, db=torch.empty(40, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.deco_weight_grad8(dy, B.packed8_empty(64, 64), dw[:, :30].contiguous())
    with pytest.raises(B.DecoError) as e:
        B.deco_weight_grad8(dy, packed, dw, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.DECO_ERR_CAPACITY


def test_rows_whose_offsets_pass_32_bits():
    """Rows of dY 2^31 entries apart, read as they are and through planes; many tiles, more than workers."""
    rows, out, cols = 3, 40, 70
    packed = checkpoint(rows, cols, 14)
    for stride in (2 ** 31 + 24, 2 ** 31 + 25):
        buf = torch.zeros((rows - 1) * stride + out, dtype=torch.bfloat16, device="cuda")
        dy = torch.as_strided(buf, (rows, out), (stride, 1))
        dy.copy_(gradients(rows, out, "bf16", 15))
        dw, db = torch.empty(out, cols, device="cuda"), torch.empty(out, device="cuda")
        B.deco_weight_grad8(dy, packed, dw, db=db)
        check(dy, packed, cols, dw, db, False)
        del buf, dy


@pytest.mark.parametrize("gtype", ["f32", "bf16"])
def test_more_tiles_than_workers_and_parts_of_many(gtype):
    """Whole tiles several to a worker; a tile in dozens of parts; blocks dealt out across tiles."""
    for rows, out, cols in ((70, 3000, 2500), (20000, 33, 50), (9000, 1500, 230)):
        packed, dy = checkpoint(rows, cols, 16), gradients(rows, out, "bf16", 17)
        dw, db = torch.empty(out, cols, device="cuda", dtype=DT[gtype]), torch.empty(out, device="cuda", dtype=DT[gtype])
        B.deco_weight_grad8(dy, packed, dw, db=db)
        check(dy, packed, cols, dw, db, False)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("lead", [16, 4])
@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,out,cols", [(70, 201, 240), (70, 129, 200), (700, 64, 1008), (9000, 700, 608)])
def test_rows_that_start_on_32_bytes_and_rows_that_do_not(rows, out, cols, gtype, lead, accumulate):
    """Whole rows of sixteen entries are written at once where they can be; what is around the matrix stays."""
    flat = torch.full((lead + out * cols + 40,), 0.5, device="cuda", dtype=DT[gtype])
    dw = flat[lead:lead + out * cols].view(out, cols)
    packed, dy = checkpoint(rows, cols, 20), gradients(rows, out, "bf16", 21)
    B.deco_weight_grad8(dy, packed, dw, accumulate=accumulate)
    check(dy, packed, cols, dw, None, False, old=0.5 if accumulate else 0.0)
    assert (flat[:lead] == 0.5).all() and (flat[lead + out * cols:] == 0.5).all()


@pytest.mark.parametrize("dtype,transposed", [("bf16", False), ("bf16", True), ("f32", False)])
def test_few_tokens_and_many_tiles(dtype, transposed):
    """Pairs of CTAs whose tiles are of one block or two of tokens."""
    for rows, out, cols in ((40, 4300, 4000), (100, 4000, 4241)):
        packed, dy = checkpoint(rows, cols, 22), gradients(rows, out, dtype, 23)
        dw, db = torch.empty((cols, out) if transposed else (out, cols), device="cuda"), torch.empty(out, device="cuda")
        B.deco_weight_grad8(dy, packed, dw, db=db, transposed=transposed)
        check(dy, packed, cols, dw, db, transposed)
