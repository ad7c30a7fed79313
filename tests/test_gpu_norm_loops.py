"""deco_layernorm and deco_layernorm_grad where every group of warps goes over many rows: slots of the rows ahead that are used again
and again, sums that change places from row to row, a last round that only some groups have.

A launch has at most 296 CTAs (of 8 entries a thread; 148 of 16 or 24), of up to 16 groups of one warp or 16 / warps of several, and up to three
rows ahead: every shape has more than seven rows for each group.  Tolerances are those of test_gpu_norm."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B
from tests.test_gpu_norm import check_grad, check_norm, gen, reference_pack, rows_of, run_norm, stats, values

pytestmark = pytest.mark.gpu

# rows, columns, entries between rows, entries before the first
SHAPES = [(40009, 200, 0, 0), (20011, 512, 0, 0), (20011, 768, 0, 0), (20011, 768, 16, 8), (9001, 1000, 0, 0), (9001, 1024, 0, 0),
          (9001, 2048, 0, 0), (2203, 4096, 0, 0), (1201, 8192, 0, 0), (40009, 201, 0, 0), (9001, 1001, 0, 0), (5003, 2048, 3, 1)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    torch.cuda.set_device(0)


def like(x, pad, lead):
    """A copy whose rows are as far apart, and start where x's do."""
    y = rows_of(x.shape[0], x.shape[1], "f32" if x.dtype == torch.float32 else "bf16", 0, pad, lead)
    return y.copy_(x)


def weights(cols):
    return 1 + 0.3 * torch.randn(cols, generator=gen(1), device="cuda"), torch.randn(cols, generator=gen(2), device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,lead", SHAPES)
def test_norm(rows, cols, pad, lead, dtype):
    w, b = weights(cols)
    x = rows_of(rows, cols, dtype, 3, pad, lead, 2.0, 0.5)
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=gen(4), device="cuda")).to(x.dtype)      # no row's statistics are another's
    add = rows_of(rows, cols, dtype, 5, pad, lead, 3.0, -1.0)
    for residual, keep in ((False, False), (False, True), (True, False), (True, True)):
        u = (x.float() + add.float()).to(x.dtype) if residual else x
        total = rows_of(rows, cols, dtype, 6, pad, lead) if residual else None
        y, mean, rstd, packed = run_norm(x, w, b, add if residual else None, total, keep=keep)
        check_norm(u, w, b, y, mean, rstd)
        assert total is None or torch.equal(total, u)
        if keep:
            q, e = reference_pack(u)
            assert torch.equal(packed[0], q) and torch.equal(packed[1], e)
    # in place: rows ahead have yet to be read.  The same bits from rows as far apart; a clone's rows lie side by side, and may be
    # summed up in another order
    for over, under, same in ((x.clone(), add.clone(), not pad), (like(x, pad, lead), like(add, pad, lead), True)):
        y2, mean, rstd, _ = run_norm(over, w, b, under, under, y=over)
        assert torch.equal(under, total)
        check_norm(total, w, b, y2, mean, rstd)
        assert torch.equal(over, y) or not same


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,lead", SHAPES)
def test_grad(rows, cols, pad, lead, dtype):
    w, _ = weights(cols)
    x = rows_of(rows, cols, dtype, 7, pad, lead, 2.0, 0.5)
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=gen(8), device="cuda")).to(x.dtype)
    mean, rstd = stats(x)
    packed = B.packed8_empty(rows, cols)
    B.deco_pack8(x, packed)
    dy, add = rows_of(rows, cols, dtype, 9, pad, lead, 1e-2), rows_of(rows, cols, dtype, 10, pad, lead, 1e-2)
    for saved, residual in ((x, False), (x, True), (packed, False), (packed, True)):
        dx = rows_of(rows, cols, dtype, 11, pad, lead)
        dw, db = torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
        B.deco_layernorm_grad(saved, mean, rstd, w, dy, dx, dweight=dw, dbias=db, add=add if residual else None)
        check_grad(x if saved is x else values(packed, cols), mean, rstd, w, dy, add if residual else None, dx, dw, db)
        over = like(dy, pad, lead)
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        B.deco_layernorm_grad(saved, mean, rstd, w, over, over, dweight=dw2, dbias=db2, add=add if residual else None)
        assert torch.equal(over, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
