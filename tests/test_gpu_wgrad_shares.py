"""deco_weight_grad8 in every way of sharing its work out: whole tiles, tiles in equal parts (two, and as many as there are), all blocks dealt
out evenly across tiles; by single CTAs and by pairs.  The workspace's size tells which it is.  Tolerances are those of test_gpu_wgrad."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B
from tests.test_gpu_wgrad import DT, check, checkpoint, gradients

pytestmark = pytest.mark.gpu

# rows, out, cols; CTAs of a worker, shares of X's columns, blocks of 64 tokens, workers, tiles
SHARES = {
    "whole tiles, several a worker, single": (70, 3000, 2500, 1, 23, 2, 0, 552),
    "whole tiles, several a worker, pairs": (64, 6000, 6000, 2, 54, 1, 0, 648),
    "two parts, pairs": (4100, 2304, 768, 2, 8, 66, 72, 36),
    "six parts, pairs": (9000, 1504, 230, 2, 4, 144, 72, 12),
    "many parts, single": (300000, 40, 50, 1, 1, 4692, 46, 1),
    "many parts, pairs": (600000, 40, 50, 2, 2, 9387, 63, 1),
    "dealt out evenly, single": (5898, 688, 468, 1, 5, 93, 148, 30),
    "dealt out evenly, pairs": (9000, 1504, 1000, 2, 10, 141, 74, 30),
}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("name", SHARES)
def test_shares(name, transposed, gtype):
    rows, out, cols, ctas, shares, blocks, workers, tiles = SHARES[name]
    packed, dy = checkpoint(rows, cols, 30), gradients(rows, out, "bf16", 31)
    # steps of 16 bytes per token and share; where tiles are cut, two parts of a tile a worker and eight counters a tile and CTA
    room = 16 * shares * blocks * 64 + (2 * workers * ctas * ctas * 128 * 128 * 4 + 4 * tiles * ctas * 8 if workers else 0)
    assert B.deco_weight_grad8_workspace(dy, cols, B.DECO_F32 if gtype == "f32" else B.DECO_BF16) == room
    dw = torch.full((cols, out) if transposed else (out, cols), 7.0, device="cuda", dtype=DT[gtype])
    db = torch.full((out,), 7.0, device="cuda", dtype=DT[gtype])
    B.deco_weight_grad8(dy, packed, dw, db=db, transposed=transposed)
    check(dy, packed, cols, dw, db, transposed)
    # whoever comes last adds the parts up, in their order: the same bits every time, whatever the workspace held
    again, b2 = torch.empty_like(dw), torch.empty_like(db)
    for _ in range(4):
        B.deco_weight_grad8(dy, packed, again.fill_(3.0), db=b2.fill_(3.0), transposed=transposed,
                            workspace=torch.randint(0, 255, (room,), dtype=torch.uint8, device="cuda"))
        assert torch.equal(again, dw) and torch.equal(b2, db)
