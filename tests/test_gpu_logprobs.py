"""deco_token_logprobs and deco_token_logprobs_grad against their definitions in 64 bits.

Tolerances.  eps = 2^-24 (fp32 rounding).  A weight 2^t carries the error of ex2 (2 eps), of t
(one rounding, |t| eps) and of the constant c = scale log2 e (|t| eps): weights with |t| > 40
vanish, so a weight's relative error is below 2 + 2 * 40 = 82 eps.  Sums over n entries held in
at least 256 partial sums add at most (n / 256 + 16) eps.  Hence

  lse       |lse| 4 eps  +  (100 + n / 256) eps                      =: |lse| 4 eps + sum_tol
  entropy   sum_tol (1 + H + 40)   (q weighs the terms by |t| <= 40)
  logprob   |lp| 4 eps + sum_tol
  gradient  |g| terms times the relative error of p: d = z - lse is rounded once on |z| + |lse|,
            so p is off by (|lse| + |z| + 8) 2 eps, plus sum_tol of the lse handed in; bf16
            outputs add half a unit in the last place, 2^-8 of the value.
"""
import math

import numpy as np
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


def sum_tol(n):
    return (100 + n / 256) * EPS


def rows_of(rows, vocab, dtype, seed, pad=0, lead=0, sigma=3.0):
    """[rows, vocab] view with `pad` entries between rows and `lead` entries before the first."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    stride = vocab + pad
    buf = torch.full((lead + rows * stride + 64,), 1e4, device="cuda", dtype=DT[dtype])
    view = buf[lead:lead + rows * stride].view(rows, stride)[:, :vocab]
    view.copy_((sigma * torch.randn(rows, vocab, generator=g, device="cuda")).to(DT[dtype]))
    return view


def call(logits, targets, top, scale=1.0, stream=None):
    rows = logits.shape[0]
    out = {k: torch.full((rows,), 77.0, device="cuda") for k in ("logprob", "entropy", "lse")}
    out["top_idx"] = torch.full((rows, top), -7, dtype=torch.int32, device="cuda")
    out["top_logprob"] = torch.full((rows, top), 77.0, device="cuda")
    B.deco_token_logprobs(logits, targets, out["logprob"], out["entropy"], out["lse"], scale,
                          out["top_idx"] if top else None, out["top_logprob"] if top else None,
                          stream=stream)
    return out


def reference(logits, targets, top, scale):
    """The definition in 64 bits; selection by a stable sort of the values as given."""
    x = logits.double()
    z = x * scale
    m = z.amax(1, keepdim=True)
    ms = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    e = torch.exp(z - ms)
    s = e.sum(1, keepdim=True)
    lse = (ms + s.log()).squeeze(1)
    lp = (z - ms) - s.log()                     # not z - lse: a row of the lowest value would lose log s
    p = lp.exp()
    h = -(torch.where(p > 0, p * lp, torch.zeros_like(p))).sum(1)
    empty = torch.isneginf(lse)
    lp[empty] = -math.inf
    h[empty] = 0
    t = targets.clamp(0, x.shape[1] - 1)
    lpt = torch.where(targets < 0, torch.zeros_like(lse), lp.gather(1, t[:, None]).squeeze(1))
    lpt = torch.where(targets >= x.shape[1], torch.full_like(lpt, math.nan), lpt)
    idx = x.sort(dim=1, descending=True, stable=True).indices[:, :top]
    return {"lse": lse, "entropy": h, "logprob": lpt, "top_idx": idx, "top_logprob": lp.gather(1, idx),
            "lp": lp, "p": p}


def close(got, want, tol):
    got, want = got.double(), want.double()
    same = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~same & ~torch.isnan(want)], want[~same & ~torch.isnan(want)])
    tol = tol if torch.is_tensor(tol) else torch.full_like(want, tol)
    bad = ((got - want).abs() > tol) & same
    assert not bad.any(), (got[bad][:4], want[bad][:4], tol[bad][:4])


def check(out, ref, vocab, top):
    st = sum_tol(vocab)
    close(out["lse"], ref["lse"], ref["lse"].abs().nan_to_num(0, 0, 0) * 4 * EPS + st)
    close(out["entropy"], ref["entropy"], st * (41 + ref["entropy"]))
    close(out["logprob"], ref["logprob"], ref["logprob"].abs().nan_to_num(0, 0, 0) * 4 * EPS + st)
    if top:
        assert torch.equal(out["top_idx"].long(), ref["top_idx"])
        close(out["top_logprob"], ref["top_logprob"], ref["top_logprob"].abs().nan_to_num(0, 0, 0) * 4 * EPS + st)


def targets_for(rows, vocab, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    t[::5] = -100
    t[0] = vocab - 1
    return t


SHAPES = [(1, 1, 0, 0), (3, 2, 0, 0), (2, 7, 1, 1), (5, 33, 3, 2), (1, 1000, 0, 0), (4, 1023, 0, 5),
          (2, 8192, 0, 0), (3, 8193, 7, 3), (1, 32000, 0, 0), (9, 32003, 0, 1), (700, 1111, 0, 0),
          (600, 4097, 1, 0), (40, 50257, 0, 0), (1, 131072, 0, 0), (2, 300001, 5, 7)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,lead", SHAPES)
def test_against_the_definition(rows, vocab, pad, lead, dtype):
    for top, scale in ((0, 1.0), (1, 0.5), (20, 1.25), (32, 1.0)):
        top = min(top, vocab)
        x = rows_of(rows, vocab, dtype, vocab + top, pad, lead)
        t = targets_for(rows, vocab, top)
        check(call(x, t, top, scale), reference(x, t, top, scale), vocab, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [37, 5000, 50257])
@pytest.mark.parametrize("rows", [2, 700])
def test_masked_rows(rows, vocab, dtype):
    """-inf, the type's lowest value and the usual finite masks: nearly everything masked, fewer
    tokens allowed than alternatives asked for, one token, none."""
    fills = [-math.inf, torch.finfo(DT[dtype]).min, -1e9, -1e4, -1e25]
    for i, fill in enumerate(fills):
        x = rows_of(rows, vocab, dtype, 7 + i)
        keep = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
        keep[:, 3::11] = True
        keep[0] = False
        keep[0, vocab - 2] = True                                  # one token left
        keep[1] = False                                            # none
        if rows > 2:
            keep[2] = False
            keep[2, ::max(1, vocab // 5)] = True                   # fewer than asked for
            keep[3] = True
            keep[3, : vocab // 2] = False                          # the first half masked
        x.masked_fill_(~keep, fill)
        top = min(20, vocab)
        t = targets_for(rows, vocab, i)
        out, ref = call(x, t, top), reference(x, t, top, 1.0)
        check(out, ref, vocab, top)


def test_equal_values_go_to_the_lower_index():
    for rows, vocab in ((1, 40000), (650, 9000)):
        for dtype in DT:
            x = rows_of(rows, vocab, dtype, 3)
            x.copy_((x * 2).round() / 2)                           # heavy ties everywhere
            x[0] = 1.5                                             # all equal
            x[-1, 1000:] = 4.0
            if rows > 1:
                x[1] = 0.0
                x[1, ::2] = -0.0                                   # +0 and -0 are one value
            t = targets_for(rows, vocab, 0)
            for top in (1, 5, 32):
                ref = reference(x, t, top, 1.0)
                if rows > 1:
                    ref["top_idx"][1] = torch.arange(top, device="cuda")
                check(call(x, t, top), ref, vocab, top)


def test_orders_that_flood_the_candidate_list():
    """Ascending rows, a block of large values at the end, and a pattern that puts all large
    values before one thread: the list of candidates overflows and the exact passes take over."""
    for rows in (1, 650):
        v = 60000
        x = torch.arange(v, device="cuda", dtype=torch.float32).repeat(rows, 1) / 3000.0
        x[0, : v // 2] = -50.0
        y = rows_of(rows, v, "f32", 5)
        lane = torch.arange(v, device="cuda") // 4 % 256 == 17
        y[:, lane] += 40.0
        for z in (x, y, x.flip(1).contiguous()):
            t = targets_for(rows, v, 2)
            for top in (1, 32):
                check(call(z, t, top), reference(z, t, top, 1.0), v, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_infinity_and_targets_out_of_range(dtype):
    for rows in (5, 800):
        v = 12345
        x = rows_of(rows, v, dtype, 9)
        x[0, 17] = math.nan
        x[1, 12000] = math.inf
        x[2] = -math.inf
        t = targets_for(rows, v, 1)
        t[0], t[1], t[2], t[3], t[4] = 5, 6, 7, v, 2 ** 40
        out = call(x, t, 3)
        for r in (0, 1):
            for k in ("lse", "entropy", "logprob"):
                assert math.isnan(out[k][r].item()), (r, k)
            assert torch.isnan(out["top_logprob"][r]).all()
        assert out["top_idx"][0, 0] == 17 and out["top_idx"][1, 0] == 12000
        assert out["lse"][2] == -math.inf and out["entropy"][2] == 0 and out["logprob"][2] == -math.inf
        assert out["top_idx"][2].tolist() == [0, 1, 2] and torch.isneginf(out["top_logprob"][2]).all()
        assert torch.isnan(out["logprob"][3:5]).all() and torch.isfinite(out["lse"][3:]).all()
        keep = [i for i in range(rows) if i > 2]
        sub = {k: o[keep] for k, o in out.items()}
        check(sub, reference(x[keep], t[keep], 3, 1.0), v, 3)


def test_extreme_scales_and_magnitudes():
    for scale in (1e-30, 1e-5, 1e5, 1e30):
        x = rows_of(3, 9001, "f32", 1)
        t = targets_for(3, 9001, 0)
        out, ref = call(x, t, 4, scale), reference(x, t, 4, float(np.float32(scale)))
        # z itself is rounded: the scaled values carry 2 eps of |z|
        z = (x.double() * scale).abs().amax(1)
        for k in ("lse", "logprob"):
            close(out[k], ref[k], z * 8 * EPS + sum_tol(9001))
        assert torch.equal(out["top_idx"].long(), ref["top_idx"])
    x = rows_of(4, 5000, "f32", 2)
    x[0] += 3e6
    x[1] *= 1e36
    x[2] -= 2e7
    t = targets_for(4, 5000, 3)
    check(call(x, t, 2), reference(x, t, 2, 1.0), 5000, 2)


def call_none(x, top):
    lse = torch.empty(x.shape[0], device="cuda")
    B.deco_token_logprobs(x, None, None, None, lse)
    return lse


def test_outputs_are_optional_and_repeatable():
    x = rows_of(33, 20011, "bf16", 4)
    t = targets_for(33, 20011, 4)
    full = call(x, t, 7)
    again = call(x, t, 7)
    for k in full:
        assert torch.equal(full[k], again[k])
    assert torch.equal(call_none(x, 0), call(x, t, 0)["lse"])
    lp = torch.empty(33, device="cuda")
    B.deco_token_logprobs(x, t, lp)
    assert torch.equal(lp, call(x, t, 0)["logprob"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = call(x, t, 7, stream=s)
    s.synchronize()
    for k in full:
        assert torch.equal(full[k], other[k])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(40, 37), (40, 9001), (700, 3001)])
@pytest.mark.parametrize("scale", [0.3, 1.5, 1.9, 1.963087797164917, 2.7261552810668945, 12.0, 200.0])
def test_masks_at_other_scales(scale, rows, vocab, dtype):
    """Finite masks of every size, which threads may see and nothing else; allowed tokens of nearly equal logits."""
    scale = float(np.float32(scale))
    for i, fill in enumerate((-1e9, -1.07e9, -3e8, -2.5e7, -3e6, -7e5, -1e4)):
        x = rows_of(rows, vocab, dtype, 13 + i, sigma=0.01)
        keep = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
        for r in range(rows):
            keep[r, r % 37::(5, 9, 40, 700)[r % 4]] = True
        keep[5] = False                                            # nothing allowed
        x.masked_fill_(~keep, fill)
        t = (torch.arange(rows, device="cuda") % 37).long()
        out, ref = call(x, t, 1, scale), reference(x, t, 1, scale)
        check(out, ref, vocab, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [300.0, -1000.0, 1e4, -5e5, 5.5e5])
def test_common_offset_of_the_logits(offset, dtype):
    """A constant added to a row changes its lse and nothing else: the tolerances are those without
    it.  Rows on one CTA and on several, whose threads and parts have different maxima."""
    for rows, scale in ((3, 1.0), (700, 1.0), (3, 1.25)):
        x = rows_of(rows, 9001, dtype, 11, sigma=2.5)
        x += offset
        t = targets_for(rows, 9001, 6)
        check(call(x, t, 8, scale), reference(x, t, 8, scale), 9001, 8)


# ------------------------------------------------------------------------------- gradient

def grads_for(rows, top, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return r(rows), r(rows), (r(rows, top) if top else None)


def grad_reference(x, t, scale, ref, idx, gl, gh, gt):
    z = torch.zeros_like(ref["p"])
    tt = torch.where(t < 0, torch.zeros_like(gl), gl).double() if gl is not None else torch.zeros(len(t), device="cuda").double()
    z.scatter_add_(1, t.clamp(0, x.shape[1] - 1)[:, None], tt[:, None])
    if gt is not None:
        z.scatter_add_(1, idx.long(), gt.double())
    dx = z - ref["p"] * z.sum(1, keepdim=True)
    if gh is not None:
        safe = torch.where(ref["p"] > 0, ref["lp"], torch.zeros_like(ref["lp"]))
        dx -= gh.double()[:, None] * ref["p"] * (safe + ref["entropy"][:, None])
    return dx * scale


def grad_tol(x, scale, ref, dtype, dx, gl, gh, gt):
    """|dx| error: relative error of p times the factor it multiplies, one rounding of the rest."""
    z = (x.double() * scale).nan_to_num(0, 0, 0).abs()
    rel = (ref["lse"].abs()[:, None] + z + 8) * 4 * EPS + sum_tol(x.shape[1])
    f = torch.zeros_like(ref["lse"])
    for g in (gl, gh):
        f = f + (g.double().abs() if g is not None else 0)
    if gt is not None:
        f = f + gt.double().abs().sum(1)
    w = f[:, None] * (1 + z + ref["lse"].abs()[:, None] + ref["entropy"][:, None])
    tol = scale * (ref["p"] * rel * w + 64 * EPS * f[:, None] * (ref["p"] + (ref["p"] > 1)) ) + dx.abs() * 40 * EPS
    return tol + (dx.abs() * 2.0 ** -8 if dtype == "bf16" else 0) + 1e-38


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,lead", SHAPES)
def test_gradient_against_the_definition(rows, vocab, pad, lead, dtype):
    for top, scale, ent, inplace in ((0, 1.0, False, False), (0, 0.7, True, True), (5, 1.25, True, False),
                                     (32, 1.0, False, True)):
        top = min(top, vocab)
        x = rows_of(rows, vocab, dtype, vocab + top, pad, lead)
        t = targets_for(rows, vocab, top)
        scale = float(np.float32(scale))
        ref = reference(x, t, top, scale)
        out = call(x, t, top, scale)
        gl, gh, gt = grads_for(rows, top, vocab)
        gh = gh if ent else None
        want = grad_reference(x, t, scale, ref, out["top_idx"], gl, gh, gt)
        tol = grad_tol(x, scale, ref, dtype, want, gl, gh, gt)
        # the target's own entry is a difference of two terms of the size of g
        own = torch.zeros_like(tol).scatter_(1, t.clamp_min(0)[:, None], 1.0)
        if top:
            own.scatter_(1, out["top_idx"].long(), 1.0)
        size = gl.abs()[:, None].double() + (gt.abs().double().sum(1, keepdim=True) if top else 0)
        tol = tol + own * size * scale * (16 * EPS + ref["p"] * (ref["lse"].abs()[:, None] + 40) * 8 * EPS)
        keep = x.clone()
        dx = x if inplace else rows_of(rows, vocab, dtype, 1, pad + 3, lead + 1)
        B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=gh,
                                   top_idx=out["top_idx"] if top else None, g_top=gt, scale=scale)
        close(dx, want, tol)
        if not inplace:
            assert torch.equal(x, keep)


def test_gradient_leaves_neighbours_alone():
    """Entries between rows, before the first and behind the last are not written."""
    for dtype in DT:
        buf = torch.full((5 + 3 * 1050 + 9,), 123.0, device="cuda", dtype=DT[dtype])
        dx = buf[5:5 + 3 * 1050].view(3, 1050)[:, :1013]
        x = rows_of(3, 1013, dtype, 1)
        t = targets_for(3, 1013, 1)
        out = call(x, t, 0)
        B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=torch.ones(3, device="cuda"))
        assert (buf[:5] == 123).all() and (buf[5 + 3 * 1050:] == 123).all()
        assert (buf[5:5 + 3 * 1050].view(3, 1050)[:, 1013:] == 123).all()
        assert (dx != 123).all()


def test_gradient_of_masked_and_ignored_rows():
    x = rows_of(6, 4001, "f32", 3)
    x[:, ::2] = -math.inf
    x[1] = -math.inf
    t = torch.tensor([1, 3, -1, 5, 4001, 7], device="cuda")
    out = call(x, t, 2)
    gl, gh, gt = grads_for(6, 2, 1)
    dx = torch.empty_like(x)
    B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl)
    assert (dx[1] == 0).all() and (dx[2] == 0).all() and torch.isnan(dx[4]).all()
    assert (dx[0, ::2] == 0).all() and (dx[0, 1::2] != 0).all()
    B.deco_token_logprobs_grad(x, t, out["lse"], dx, entropy=out["entropy"], g_entropy=gh, top_idx=out["top_idx"],
                               g_top=gt)
    assert torch.isfinite(dx).all() and (dx[1] == 0).all()
    # every row of a log-softmax gradient sums to zero: within the roundings of its entries
    tol = dx.abs().double().sum(1) * 64 * EPS + sum_tol(4001) * 100
    assert (dx.double().sum(1).abs() <= tol).all()


def test_gradient_against_differences():
    """Central differences of the 64-bit value: h = 2^-10, error h^2 |f'''| / 6 <= 2^-20 on terms of size
    1, far above the fp32 roundings."""
    x = rows_of(2, 300, "f32", 8, sigma=1.0)
    t = torch.tensor([17, 250], device="cuda")
    out = call(x, t, 3, 1.25)
    gl, gh, gt = grads_for(2, 3, 5)
    dx = torch.empty_like(x)
    B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=gh,
                               top_idx=out["top_idx"], g_top=gt, scale=1.25)

    def value(y):
        lp = torch.log_softmax(y * 1.25, 1)
        return (gl.double() * lp.gather(1, t[:, None])[:, 0]).sum() - (gh.double() * (lp.exp() * lp).sum(1)).sum() + \
            (gt.double() * lp.gather(1, out["top_idx"].long())).sum()
    h = 2.0 ** -10
    for r, j in ((0, 17), (0, 3), (1, 250), (1, int(out["top_idx"][1, 0])), (0, 299)):
        y = x.double()
        y[r, j] += h
        up = value(y)
        y[r, j] -= 2 * h
        want = ((up - value(y)) / (2 * h)).item()
        assert abs(dx[r, j].item() - want) < 2e-5


def grad_from_lse(x, t, scale, lse, entropy, idx, gl, gh, gt):
    """The formula in 64 bits with p = exp(z - lse) of the lse as given; and p."""
    z = x.double() * scale
    lp = z - lse.double()[:, None]
    ref = {"p": lp.exp(), "lp": lp, "entropy": entropy.double()}
    return grad_reference(x, t, scale, ref, idx, gl, gh, gt), ref["p"]


@pytest.mark.parametrize("ent", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0.0, 300.0, -1e4, 5e5])
def test_gradient_follows_the_lse_it_is_given(offset, dtype, ent):
    """p = exp(z - lse) for the lse handed in, which is exact here whatever its size: a weight's error
    is that of a sum without an offset (82 eps and 20 for the row's factor), times what it multiplies.
    Logits more than 40 below lse have p < 2^-57 and do not show."""
    rows, v, top = 5, 9001, 4
    for scale in (1.0, 1.25, 0.3):
        scale = float(np.float32(scale))
        x = rows_of(rows, v, dtype, 21, sigma=2.5)
        x += offset
        t = targets_for(rows, v, 3)
        out = call(x, t, top, scale)
        gl, gh, gt = grads_for(rows, top, 8)
        gh = gh if ent else None
        want, p = grad_from_lse(x, t, scale, out["lse"], out["entropy"], out["top_idx"], gl, gh, gt)
        f = gl.abs().double() + gt.abs().double().sum(1)
        w = f[:, None] + (gh.abs().double() * (41 + out["entropy"].double()) if ent else 0 * f)[:, None]
        own = torch.zeros_like(want).scatter_(1, t.clamp_min(0)[:, None], 1.0).scatter_(1, out["top_idx"].long(), 1.0)
        tol = scale * (102 * EPS * p * w + 16 * EPS * own * f[:, None]) + want.abs() * 2.0 ** (-8 if dtype == "bf16" else -23)
        dx = torch.empty_like(x)
        B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=gh,
                                   top_idx=out["top_idx"], g_top=gt, scale=scale)
        close(dx, want, tol + 1e-36)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(6, 37), (6, 50257), (150, 9001)])
def test_gradient_of_rows_whose_lse_has_lost_its_last_digits(rows, vocab, dtype, inplace):
    """Rows of the type's lowest value or another finite mask alone, and logits of 1e7 and more: the spacing of
    fp32 there is larger than log(vocab), so an lse does not tell one token from all.  With z - max exact (these
    logits and scales) p is off by that of expf and the sum: 8 eps, |z - max| eps, |log sum| eps, sum_tol."""
    lowest = torch.finfo(DT[dtype]).min
    for scale in (1.0, 2.0):                                       # twice the lowest value overflows
        x = rows_of(rows, vocab, dtype, 31, pad=3, lead=1)
        x[0], x[1], x[2] = lowest, -1e9, -1e25
        x[3] = lowest
        x[3, 3::7] = -3e8                                          # a few above the others, equal
        x[4] = 2.0 ** 24 * (1 + torch.arange(vocab, device="cuda") % 3)
        x[5] = -math.inf
        t = targets_for(rows, vocab, 2)
        t[:6] = torch.tensor([2, vocab - 1, -1, 3, 5, 1], device="cuda")
        top = 3
        out, ref = call(x, t, top, scale), reference(x, t, top, scale)
        gl, gh, gt = grads_for(rows, top, 5)
        keep = slice(0, 5)
        for g_h in (None, gh):
            want = grad_reference(x, t, scale, ref, ref["top_idx"], gl, g_h, gt)[keep]
            f = (gl.abs().double() + gt.abs().double().sum(1))[keep, None]
            h = ref["entropy"][keep, None]
            w = f + (gh.abs().double()[keep, None] * (41 + h) if g_h is not None else 0)
            own = torch.zeros_like(want).scatter_(1, t[keep].clamp_min(0)[:, None], 1.0)
            own.scatter_(1, out["top_idx"][keep].long(), 1.0)
            p = ref["p"][keep]
            tol = scale * (((50 + h) * 2 * EPS + 2 * sum_tol(vocab)) * p * w + 16 * EPS * own * f)
            tol = tol + want.abs() * 2.0 ** (-8 if dtype == "bf16" else -23)
            logits = x.clone() if inplace else x
            dx = logits if inplace else torch.empty_like(x)
            B.deco_token_logprobs_grad(logits, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=g_h,
                                       top_idx=out["top_idx"], g_top=gt, scale=scale)
            close(dx[keep], want, tol + 1e-38)
            assert (dx[5] == 0).all()
            if rows > 6:                                           # ordinary rows of the same call
                assert torch.isfinite(dx[6:]).all() and (dx[6:] != 0).any(1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-5, 300.0, 1e4, 1e30])
def test_gradient_at_unusual_scales(scale, dtype):
    """Scales outside [2^-8, 2^8].  Below |lse| = 2^20 ln 2 p follows the lse handed in: d = z - lse rounded once,
    exp of it: |d| eps and 8 eps.  Beyond it, (x - max) scale is rounded once, as above."""
    rows, v, top = 4, 5003, 3
    scale = float(np.float32(scale))
    x = rows_of(rows, v, dtype, 41)
    t = targets_for(rows, v, 4)
    out, ref = call(x, t, top, scale), reference(x, t, top, scale)
    gl, gh, gt = grads_for(rows, top, 6)
    if ref["lse"].abs().max() < 2.0 ** 20 * math.log(2.0) - 1:
        want, p = grad_from_lse(x, t, scale, out["lse"], out["entropy"], out["top_idx"], gl, gh, gt)
        h = out["entropy"].double()[:, None]
    else:
        want, p, h = grad_reference(x, t, scale, ref, ref["top_idx"], gl, gh, gt), ref["p"], ref["entropy"][:, None]
    f = (gl.abs().double() + gt.abs().double().sum(1))[:, None]
    w = f + gh.abs().double()[:, None] * (41 + h)
    own = torch.zeros_like(want).scatter_(1, t.clamp_min(0)[:, None], 1.0).scatter_(1, out["top_idx"].long(), 1.0)
    tol = scale * (((50 + h) * 2 * EPS + 2 * sum_tol(v)) * p * w + 16 * EPS * own * f)
    tol = tol + want.abs() * 2.0 ** (-8 if dtype == "bf16" else -23) + 1e-38
    dx = torch.empty_like(x)
    B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=gh,
                               top_idx=out["top_idx"], g_top=gt, scale=scale)
    close(dx, want, tol)


@pytest.mark.parametrize("offset", [0.0, 2e7])
def test_gradient_of_repeated_and_left_out_alternatives(offset):
    """Equal tokens among the alternatives and the target add up; indices >= vocab are left out."""
    rows, v = 3, 6007
    x = rows_of(rows, v, "f32", 51) * 8 + offset
    t = torch.tensor([17, 6006, -1], device="cuda")
    idx = torch.tensor([[17, 17, 4, 6007, 17], [0, 6006, 0, -1, 2 ** 31 - 1], [5, 5, 5, 5, 5]], dtype=torch.int32,
                       device="cuda")
    out, ref = call(x, t, 0), reference(x, t, 0, 1.0)
    gl, _, gt = grads_for(rows, 5, 7)
    inside = (idx >= 0) & (idx < v)
    want = grad_reference(x, t, 1.0, ref, torch.where(inside, idx, torch.zeros_like(idx)), gl, None,
                          torch.where(inside, gt, torch.zeros_like(gt)))
    f = (gl.abs().double() + gt.abs().double().sum(1))[:, None]
    tol = (ref["p"] * (ref["lse"].abs()[:, None] * (4 if offset == 0 else 0) + 60) * 2 * EPS + 2 * sum_tol(v) * ref["p"] + 16 * EPS) * f
    dx = torch.empty_like(x)
    B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, top_idx=idx, g_top=gt)
    close(dx, want, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_of_rows_with_nan_or_infinity(dtype):
    """lse is NaN there, and so is the gradient; a row of -inf has the gradient 0, also where its target is not one."""
    for rows, v in ((5, 37), (400, 9001)):
        x = rows_of(rows, v, dtype, 81)
        x[0, 5], x[1, v - 1], x[2], x[3] = math.nan, math.inf, -math.inf, -math.inf
        t = targets_for(rows, v, 1)
        t[3] = v
        out = call(x, t, 2)
        gl, gh, gt = grads_for(rows, 2, 3)
        for g_h in (None, gh):
            dx = torch.empty_like(x)
            B.deco_token_logprobs_grad(x, t, out["lse"], dx, g_logprob=gl, entropy=out["entropy"], g_entropy=g_h,
                                       top_idx=out["top_idx"], g_top=gt)
            assert torch.isnan(dx[:2]).all() and (dx[2:4] == 0).all() and torch.isfinite(dx[4:]).all()


def test_rows_whose_offsets_pass_32_bits():
    """Rows 2^31 + 2^29 entries apart, outputs and gradient (in place) against the definition."""
    v, stride, rows = 4001, 2 ** 31 + 2 ** 29 + 3, 3
    buf = torch.zeros(2 * stride + v + 8, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (rows, v), (stride, 1), 1)
    x.copy_(rows_of(rows, v, "bf16", 61))
    t = targets_for(rows, v, 5)
    out, ref = call(x, t, 4), reference(x, t, 4, 1.0)
    check(out, ref, v, 4)
    gl, gh, gt = grads_for(rows, 4, 9)
    want, p = grad_from_lse(x, t, 1.0, out["lse"], out["entropy"], out["top_idx"], gl, gh, gt)
    f = gl.abs().double() + gt.abs().double().sum(1)
    w = f[:, None] + (gh.abs().double() * (41 + out["entropy"].double()))[:, None]
    own = torch.zeros_like(want).scatter_(1, t.clamp_min(0)[:, None], 1.0).scatter_(1, out["top_idx"].long(), 1.0)
    B.deco_token_logprobs_grad(x, t, out["lse"], x, g_logprob=gl, entropy=out["entropy"], g_entropy=gh,
                               top_idx=out["top_idx"], g_top=gt)
    close(x, want, 102 * EPS * p * w + 16 * EPS * own * f[:, None] + want.abs() * 2.0 ** -8 + 1e-36)
    assert (buf[0] == 0) and (buf[1 + v:1 + stride] == 0).all() and (buf[-7:] == 0).all()


def test_the_longest_row():
    """vocab = 2^31 - 1, bf16, one entry off a 16-byte boundary.  Sums of n entries in 2048 threads: 82 eps for a
    weight and n / 2048 / 2 eps for sums of equal terms are too much to ask for; their roundings are spread, so
    sqrt(n / 2048) of them: 1024 eps."""
    v = 2 ** 31 - 1
    buf = torch.zeros(v + 16, dtype=torch.bfloat16, device="cuda")
    x = buf[1:1 + v].view(1, v)
    step = 2 ** 28
    g = torch.Generator(device="cuda")
    g.manual_seed(71)
    for lo in range(0, v, step):
        n = min(step, v - lo)
        x[0, lo:lo + n] = torch.randn(n, generator=g, device="cuda", dtype=torch.bfloat16)
    spots = [0, 6, 7, 2 ** 30 + 5, 2 ** 31 - 10, v - 1]
    for i, j in enumerate(spots):
        x[0, j] = 9.0 - i // 2                                     # the largest, in pairs of equal ones
    t = torch.tensor([v - 1], device="cuda")
    out = call(x, t, 6)
    assert out["top_idx"][0].tolist() == spots
    m, s, q = 9.0, 0.0, 0.0
    for lo in range(0, v, step):
        z = x[0, lo:lo + step].double() - m
        p = z.exp()
        s += p.sum().item()
        q += (p * z).sum().item()
        del z, p
    lse, entropy = m + math.log(s), math.log(s) - q / s
    tol = 1200 * EPS
    assert abs(out["lse"].item() - lse) <= tol + 4 * EPS * lse
    assert abs(out["entropy"].item() - entropy) <= tol * (41 + entropy)
    assert abs(out["logprob"].item() - (7.0 - lse)) <= tol + 4 * EPS * lse
    gl = torch.ones(1, device="cuda")
    keep = {j: x[0, j].item() for j in spots + [12345, 2 ** 31 - 3]}
    B.deco_token_logprobs_grad(x, t, out["lse"], x, g_logprob=gl)
    for j, z in keep.items():
        want = (1.0 if j == v - 1 else 0.0) - math.exp(z - out["lse"].item())
        assert abs(x[0, j].item() - want) <= abs(want) * (2.0 ** -8 + 200 * EPS) + 16 * EPS * (j == v - 1)
    assert buf[0] == 0 and (buf[1 + v:] == 0).all()


# ------------------------------------------------------------------------------- refusals

def test_refusals():
    x = torch.randn(4, 100, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    lp = torch.empty(4, device="cuda")
    idx = lambda k: torch.empty(4, k, dtype=torch.int32, device="cuda")  # noqa: E731
    val = lambda k: torch.empty(4, k, device="cuda")  # noqa: E731
    wide = torch.randn(4, 20, device="cuda")

    def status(fn, *a, **k):
        with pytest.raises(B.DecoError) as e:
            fn(*a, **k)
        return e.value.status
    assert status(B.deco_token_logprobs, x, t, lp, top_idx=idx(33), top_logprob=val(33)) == B.DECO_ERR_CAPACITY
    assert status(B.deco_token_logprobs, wide, t, lp, top_idx=idx(21), top_logprob=val(21)) == B.DECO_ERR_INVALID_ARG
    assert status(B.deco_token_logprobs, x, None, lp) == B.DECO_ERR_INVALID_ARG
    assert status(B.deco_token_logprobs, x, t, None) == B.DECO_ERR_INVALID_ARG
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert status(B.deco_token_logprobs, x, t, lp, scale=scale) == B.DECO_ERR_INVALID_ARG
        assert status(B.deco_token_logprobs_grad, x, t, lp, torch.empty_like(x), g_logprob=lp,
                      scale=scale) == B.DECO_ERR_INVALID_ARG
    assert status(B.deco_token_logprobs, x, t, lp, top_idx=idx(2)) == B.DECO_ERR_INVALID_ARG
    g = torch.empty_like(x)
    assert status(B.deco_token_logprobs_grad, x, t, None, g, g_logprob=lp) == B.DECO_ERR_INVALID_ARG
    assert status(B.deco_token_logprobs_grad, x, None, lp, g, g_logprob=lp) == B.DECO_ERR_INVALID_ARG
    assert status(B.deco_token_logprobs_grad, x, t, lp, g, g_entropy=lp) == B.DECO_ERR_INVALID_ARG
    for bad in (x.half(), x.t(), x[0], x.double()):
        with pytest.raises(ValueError):
            B.deco_token_logprobs(bad, t, lp)
    with pytest.raises(ValueError):
        B.deco_token_logprobs(x, t.int(), lp)
    with pytest.raises(ValueError):
        B.deco_token_logprobs(x, t, lp[:3])
    with pytest.raises(ValueError):                                # a broadcast gradient is not a buffer of 4
        B.deco_token_logprobs_grad(x, t, lp, g, g_logprob=torch.ones(1, device="cuda").expand(4))
    B.deco_token_logprobs(x[:0], t[:0], lp[:0])                    # no rows: nothing to do
    lib = B.load()
    assert lib.deco_token_logprobs(x.data_ptr() + 1, B.DECO_F32, 1, 10, 10, t.data_ptr(), 1.0, lp.data_ptr(), None,
                                   None, 0, None, None, None) == B.DECO_ERR_INVALID_ARG
    assert lib.deco_token_logprobs(x.data_ptr(), 7, 1, 10, 10, t.data_ptr(), 1.0, lp.data_ptr(), None, None, 0,
                                   None, None, None) == B.DECO_ERR_INVALID_ARG
    assert lib.deco_token_logprobs(x.data_ptr(), B.DECO_F32, 2, 10, 9, t.data_ptr(), 1.0, lp.data_ptr(), None, None,
                                   0, None, None, None) == B.DECO_ERR_INVALID_ARG
