"""deco_weight_grad8 over many tokens: sums of one sign, where what is cut off adds up.

Tolerances.  eps = 2^-24, S = sum_t |dy_t x_t|.  The tensor cores cut sums off at 2^-23 of the sum at each addition of 16
tokens.  Whatever the number of tokens, such a sum is over at most 2048 of them (512 where the result is fp32), and once more for
each further plane of fp32 dy: 256 eps S a plane; these sums are joined by rounded additions, at most rows / 512 (fp32) or rows / 2048
(bf16) of them, eps S each.  fp32 dy in two planes loses 2^-17 of each term.  A bf16 result is then off by half its own unit.

  fp32 result    (192 + rows / 512) eps S
  bf16 result    (256 planes + rows / 2048) eps S + 2^-17 S (fp32 dy) + half a unit
"""
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
    yield
    torch.cuda.empty_cache()


def half_unit(v):
    """Half the distance of the bf16 numbers around v: v = f 2^e, f in [1/2, 1), eight bits of f."""
    return torch.ldexp(torch.ones_like(v), torch.frexp(v).exponent - 9)


# more tiles than workers and not many, so that one accumulator's range is nearly all tokens
@pytest.mark.parametrize("rows,dtype,gtype", [(1 << 20, "bf16", "bf16"), (1 << 19, "f32", "bf16"), (1 << 18, "bf16", "f32")])
def test_sums_of_one_sign(rows, dtype, gtype):
    out, cols, part = 2304, 2016, 1 << 16
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    packed = B.packed8_empty(rows, cols)
    packed[1].fill_(120)
    dy = torch.empty(rows, out, device="cuda", dtype=DT[dtype])
    scale = 2.0 ** torch.linspace(0, 1, out, device="cuda")       # every part of a unit's range
    want = torch.zeros(out, cols, device="cuda", dtype=torch.float64)
    total = torch.zeros(out, device="cuda", dtype=torch.float64)
    for t in range(0, rows, part):
        packed[0][t:t + part] = torch.randint(1, 128, (part, cols), generator=g, device="cuda", dtype=torch.int8)
        dy[t:t + part] = (0.5 + torch.rand(part, out, generator=g, device="cuda")) * scale
        here = dy[t:t + part].double()
        want += here.t() @ (packed[0][t:t + part].double() * 2.0 ** -7)
        total += here.sum(0)
    dw, db = torch.empty(out, cols, device="cuda", dtype=DT[gtype]), torch.empty(out, device="cuda", dtype=DT[gtype])
    B.deco_weight_grad8(dy, packed, dw, db=db)
    if gtype == "f32":
        loss = (192 + rows / 512) * EPS
    else:
        loss = (256 * (2 if dtype == "f32" else 1) + rows / 2048) * EPS + (2.0 ** -17 if dtype == "f32" else 0)
    for got, want in ((dw, want), (db, total)):
        tol = loss * want + (half_unit(want * (1 + loss)) if gtype == "bf16" else EPS * want)
        worst = ((got.double() - want).abs() / tol).max().item()
        assert worst <= 1.0, "%.3g of the tolerance" % worst
