"""deco_orth_*: orthogonalised updates against the polynomial in 64 bits.

Tolerance in the 2-norm of a matrix.  bf16 outputs: rounding errors uniform within half a unit, 2^-9 to
2^-8 of a value: 1.7e-3 on average over many entries, at most 2^-8 = 3.9e-3 for one.  Products: each
step rounds A, P and the operand X to 11 bits (2^-12 on average 0.42 * 2^-11 = 2.0e-4 of a value); a
rounding of step i reaches the output through the steps behind it, whose mean slope is below 1.5,
and b A and c A^2 (up to 4.8 and 2.0 times A, of opposite sign) cancel: 5 steps x 3 roundings x about 3
added in squares, 2.0e-4 * 3 * sqrt(15) = 2.4e-3 at most.  Together sqrt(1.7^2 + 2.4^2) e-3 = 2.9e-3;
4e-3 is asked for, and 6.5e-3 (2^-8 more or less whole) where a matrix has fewer than 64 entries.
Momentum is one fused multiply-add: 2^-24 of its terms.
"""
import math

import pytest
import torch

from paper_2507_17346_b200 import binding as B

gpu = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    if torch.cuda.is_available():
        torch.cuda.set_device(0)


def exact(y, steps=5, coef=None, eps=1e-7):
    coef = coef or [COEF] * steps
    x = y.double()
    x = x / (x.norm() + eps)
    if x.shape[0] > x.shape[1]:
        return exact_wide(x.t(), coef).t()
    return exact_wide(x, coef)


def exact_wide(x, coef):
    for a, b, c in coef:
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def tol(numel):
    return 6.5e-3 if numel < 64 else 4e-3


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def make(rows, cols, kind, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = r(rows, cols)
    if kind == "outlier":
        x[:: max(2, rows // 7)] *= 50
    elif kind == "rank1":
        x = r(rows, 1) @ r(1, cols)
    elif kind == "lowrank":
        x = r(rows, 4) @ r(4, cols) + 1e-3 * x
    elif kind == "sparse":
        x = torch.where(x.abs() > 2.2, x, torch.zeros_like(x))
        x[rows // 2, cols // 2] = 3.0
    elif kind == "tiny":
        x = x * 1e-3
    return (0.02 * x).to(dtype)


def run_one(x, **kw):
    """x laid in a flat vector with a few entries around it, which must stay as they are."""
    n = x.numel()
    flat = torch.full((n + 11,), 5.0, device="cuda", dtype=x.dtype)
    flat[3:3 + n] = x.reshape(-1)
    out = torch.full((n + 11,), -9.0, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(n + 11, [(3, x.shape[0], x.shape[1])], **kw)
    try:
        B.deco_orth_run(h, flat, out)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)
    assert (out[:3] == -9).all() and (out[3 + n:] == -9).all()
    return out[3:3 + n].view(x.shape)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (5, 5), (8, 64), (64, 8), (63, 65), (64, 147), (147, 64), (128, 128), (129, 127),
          (130, 1000), (1000, 130), (255, 257), (256, 512), (300, 301), (384, 640), (640, 385), (513, 1100), (1025, 520),
          # one launch for all steps: one to eight CTAs, one to five tiles each, either orientation; and just beyond
          (17, 500), (3, 5000), (5000, 3), (64, 5120), (5120, 61), (64, 5121), (128, 1024), (1024, 127), (65, 900),
          (128, 1025), (100, 1300), (1300, 100), (60, 6000), (200, 3000)]


@gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shapes(rows, cols, dtype):
    x = make(rows, cols, "normal", rows * 7 + cols, dtype)
    got = run_one(x)
    assert rel(got, exact(x)) < tol(x.numel())


@gpu
@pytest.mark.parametrize("rows,cols", [(48, 100), (48, 1500), (1500, 41), (80, 128), (80, 1000), (1000, 72), (112, 250),
                                       (97, 1024), (1024, 111), (176, 3000), (208, 176)])
def test_short_sides_that_are_no_multiple_of_a_warp(rows, cols):
    """Lanes beyond the short side leave the kernels' loops early: one to eight CTAs, and the general way."""
    x = make(rows, cols, "normal", rows + cols)
    first = run_one(x)
    assert rel(first, exact(x)) < tol(x.numel())
    for _ in range(3):
        assert torch.equal(run_one(x), first)


@gpu
@pytest.mark.parametrize("kind", ["outlier", "rank1", "lowrank", "sparse", "tiny"])
@pytest.mark.parametrize("rows,cols", [(96, 200), (520, 260), (700, 768)])
def test_spectra(rows, cols, kind):
    """Spectra that gradients have; in rank 1 and rank 4 the missing directions must stay empty."""
    x = make(rows, cols, kind, rows + cols)
    assert rel(run_one(x), exact(x)) < tol(x.numel())


@gpu
@pytest.mark.parametrize("steps,coef", [(1, None), (2, None), (3, None), (8, None), (5, (2.0, -1.5, 0.5)),
                                        (4, [(3.0, -3.2, 1.2), (2.5, -2.5, 1.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]),
                                        (4, [(8.2, -23.5, 17.2), (4.1, -2.9, 0.54), (3.9, -2.8, 0.53), (2.0, -1.5, 0.5)])])
def test_steps_and_coefficients(steps, coef):
    x = make(200, 333, "normal", steps)
    each = [COEF] * steps if coef is None else coef if isinstance(coef, list) else [coef] * steps
    got = run_one(x, steps=steps, coef=coef)
    # more steps carry more roundings: their squares add up; roundings of A and P enter with the size
    # of the terms that cancel, |a| + |b| + |c|, 10.25 for the standard coefficients
    steep = max(1.0, max(sum(abs(v) for v in c) for c in each) / 10.25)
    bound = tol(x.numel()) if steep == 1.0 else math.hypot(1.7e-3, 2.4e-3 * steep)
    assert rel(got, exact(x, steps, each)) < bound * math.sqrt(max(1.0, steps / 5))


@gpu
@pytest.mark.parametrize("scale", [0, 1, 2])
def test_output_scale(scale):
    for rows, cols in ((260, 100), (100, 260)):
        x = make(rows, cols, "normal", 3)
        s = {0: 1.0, 1: math.sqrt(max(1.0, rows / cols)), 2: 0.2 * math.sqrt(max(rows, cols))}[scale]
        assert rel(run_one(x, scale=scale), s * exact(x)) < tol(x.numel())


@gpu
def test_extreme_norms_zero_and_nan():
    x = make(70, 90, "normal", 1)
    for f in (1e30, 1e-30, 3e37):
        y = x * f
        assert rel(run_one(y, eps=1e-38), exact(y, eps=1e-38)) < tol(x.numel())
    small = x * 1e-8                                                # eps takes part
    assert rel(run_one(small), exact(small)) < tol(x.numel())
    assert (run_one(torch.zeros_like(x)) == 0).all()
    bad = x.clone()
    bad[3, 4] = math.nan
    assert torch.isnan(run_one(bad)).all()
    bad[3, 4] = math.inf
    assert torch.isnan(run_one(bad)).any()


def flat_case(shapes, gap, dtype, seed):
    mats, at = [], gap
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c + gap
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return mats, at, torch.randn(at, generator=g, device="cuda").mul_(0.02).to(dtype)


MANY = [(64, 147), (64, 576), (1, 64), (128, 64), (300, 100), (100, 300), (257, 129), (40, 2100), (2100, 40), (512, 256)]


@gpu
@pytest.mark.parametrize("workspace", [0, 1, 1_000_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_matrices_with_momentum(dtype, workspace):
    """Matrices of many shapes in one handle, in one group and in several; two passes with momentum."""
    for nesterov in (False, True):
        mats, d, x = flat_case(MANY, 5, dtype, 11)
        m = torch.randn(d, device="cuda") * 0.05
        out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
        h = B.deco_orth_init(d, mats, momentum=0.9, nesterov=nesterov, workspace_bytes=workspace)
        try:
            for _ in range(2):
                want = m.double() * float(torch.tensor(0.9)) + x.double()
                B.deco_orth_run(h, x, out, momentum=m)
                bound = (want.abs() + x.double().abs()) * 2.0 ** -23 + 1e-38
                assert ((m.double() - want).abs() <= bound).all()   # entries of no matrix too
                y = m.double() * float(torch.tensor(0.9)) + x.double() if nesterov else m.double()
                used = torch.zeros(d, dtype=torch.bool, device="cuda")
                for at, r, c in mats:
                    used[at:at + r * c] = True
                    assert rel(out[at:at + r * c].view(r, c), exact(y[at:at + r * c].view(r, c))) < tol(r * c)
                assert (out[~used] == -9).all()
            st = B.deco_orth_get_stats(h)
            assert st["device_status"] == 0 and st["groups"] == (1 if workspace == 0 else st["groups"])
            assert workspace == 0 or st["groups"] > 1
        finally:
            B.deco_orth_destroy(h)


@gpu
def test_row_strides_and_interleaved_columns():
    """Three matrices that are column ranges of one buffer of rows, a strided one, and plain ones between."""
    S = 700
    mats = [(10, 120, 200, S), (10 + 200, 120, 300, S), (10 + 500, 120, 190, S), (10 + 120 * S, 33, 77)]
    d = 10 + 120 * S + 33 * 77 + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn(d, generator=g, device="cuda")
    for momentum in (False, True):
        m = torch.randn(d, device="cuda") if momentum else None
        out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
        h = B.deco_orth_init(d, mats, momentum=0.5)
        try:
            y = m.double() * 0.5 + x.double() if momentum else x.double()
            B.deco_orth_run(h, x, out, momentum=m)
            if momentum:
                assert ((m.double() - y).abs() <= (y.abs() + x.double().abs()) * 2.0 ** -23).all()
            used = torch.zeros(d, dtype=torch.bool, device="cuda")
            for q in mats:
                s = q[3] if len(q) > 3 else q[2]
                pick = lambda t: torch.as_strided(t, (q[1], q[2]), (s, 1), q[0])  # noqa: E731
                pick(used).fill_(True)
                assert rel(pick(out), exact(pick(y))) < tol(q[1] * q[2])
            assert (out[~used] == -9).all()
        finally:
            B.deco_orth_destroy(h)


@gpu
def test_same_bits_again_and_on_another_stream():
    mats, d, x = flat_case(MANY, 0, torch.float32, 3)
    outs = []
    h = B.deco_orth_init(d, mats)
    s = torch.cuda.Stream()
    try:
        for stream in (None, None, s):
            out = torch.zeros(d, device="cuda", dtype=torch.bfloat16)
            s.wait_stream(torch.cuda.current_stream())
            B.deco_orth_run(h, x, out, stream=stream)
            torch.cuda.synchronize()
            outs.append(out)
        # handles that come and go in the same memory
        B.deco_orth_destroy(h)
        h = B.deco_orth_init(d, list(reversed(mats)))
        out = torch.zeros(d, device="cuda", dtype=torch.bfloat16)
        B.deco_orth_run(h, x, out)
        torch.cuda.synchronize()
        outs.append(out)
    finally:
        B.deco_orth_destroy(h)
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


@gpu
def test_larger_than_one_wave():
    """More tiles than SMs, several tiles per CTA, long products."""
    mats, d, x = flat_case([(1100, 2300), (2300, 1100), (1000, 1000), (200, 5000)], 0, torch.bfloat16, 5)
    out = torch.zeros(d, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(d, mats)
    try:
        B.deco_orth_run(h, x, out)
        for at, r, c in mats:
            assert rel(out[at:at + r * c].view(r, c), exact(x[at:at + r * c].view(r, c))) < tol(r * c)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)


@gpu
@pytest.mark.parametrize("delta,tau", [(0.01, 0), (0.01, 2), (0.5, 1)])
def test_server_update(delta, tau):
    """deco_apply_update_orth in the iteration: sparse and dense aggregates, momentum, weight decay."""
    shapes, gap, n, lr, wd, mu = [(64, 147), (300, 100), (129, 257)], 13, 3, 0.02, 0.1, 0.9
    mats, d, _ = flat_case(shapes, gap, torch.float32, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    params = (0.05 * torch.randn(d, generator=g, device="cuda")).contiguous()
    want = params.double().clone()
    ctx = B.deco_init(d, n, delta, tau, lr, lr_at_server=True, params=params)
    h = B.deco_orth_init(d, mats, momentum=mu, scale=B.DECO_ORTH_SCALE_RMS)
    m = torch.zeros(d, device="cuda")
    wm = torch.zeros(d, device="cuda", dtype=torch.float64)
    sums = []
    mu32, lr32, w32 = (float(torch.tensor(v)) for v in (mu, lr, 1.0 / n))
    decay = float(torch.tensor(1.0) - torch.tensor(lr) * torch.tensor(wd))
    try:
        for t in range(5):
            B.deco_ef_compress(ctx, torch.randn(n, d, generator=g, device="cuda"))
            with pytest.raises(B.DecoError):
                B.deco_apply_update_orth(ctx, h, m, wd)             # out of order
            B.deco_aggregate_stale(ctx)
            k, buf = B.deco_get_k(ctx), B.deco_get_buffers(ctx)
            pairs = B.view_i32(buf["msg"], (n, buf["k_cap"], 2))[:, :k]
            s = torch.zeros(d, device="cuda", dtype=torch.float64)
            for i in range(n):
                s.index_add_(0, pairs[i, :, 0].long(), pairs[i, :, 1].contiguous().view(torch.float32).double())
            sums.append(s)
            B.deco_apply_update_orth(ctx, h, m, wd)
            if t < tau:
                continue
            wm = mu32 * wm + w32 * sums[t - tau]
            used = torch.zeros(d, dtype=torch.bool, device="cuda")
            step = torch.zeros(d, device="cuda", dtype=torch.float64)
            for at, r, c in mats:
                used[at:at + r * c] = True
                step[at:at + r * c] = (0.2 * math.sqrt(max(r, c)) * exact(wm[at:at + r * c].view(r, c))).reshape(-1)
            want = want * decay - lr32 * torch.where(used, step, wm)
            # momentum: three fp32 roundings of terms of its size, five passes
            assert (m.double() - wm).norm() <= 20 * 2.0 ** -24 * (wm.norm() + sum(x.norm() for x in sums))
            # parameters of matrices: the products' share of the tolerance on each of the t + 1 updates
            err = (params.double() - want)
            assert err[used].norm() <= 2.9e-3 * lr32 * step[used].norm() * (t + 1) + 1e-6 * want.norm()
            assert err[~used].norm() <= 1e-6 * want.norm()
        assert B.deco_get_stats(ctx)["step"] == 5 and B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)
        B.deco_destroy(ctx)


@gpu
def test_server_update_refusals():
    d = 4096
    m = torch.zeros(d, device="cuda")
    plain = B.deco_init(d, 1, 0.1, 0, 0.1)
    server = B.deco_init(d, 1, 0.1, 0, 0.1, lr_at_server=True)
    good, other = B.deco_orth_init(d, [(0, 64, 64)]), B.deco_orth_init(d + 1, [(0, 64, 64)])
    strided, nest = B.deco_orth_init(d, [(0, 32, 64, 128)]), B.deco_orth_init(d, [(0, 64, 64)], nesterov=True)
    try:
        for ctx in (plain, server):
            B.deco_ef_compress(ctx, torch.randn(1, d, device="cuda"))
            B.deco_aggregate_stale(ctx)
        for ctx, h, mom in ((plain, good, m), (server, strided, m), (server, nest, m),
                            (server, other, torch.zeros(d + 1, device="cuda"))):
            with pytest.raises(B.DecoError) as e:
                B.deco_apply_update_orth(ctx, h, mom)
            assert e.value.status == B.DECO_ERR_INVALID_ARG
        with pytest.raises(B.DecoError):
            B.deco_apply_update_orth(server, good, m, weight_decay=-1.0)
        with pytest.raises(ValueError):
            B.deco_apply_update_orth(server, good, torch.zeros(d - 1, device="cuda"))
        B.deco_apply_update_orth(server, good, m)                   # a refusal changed nothing
        B.deco_apply_update(plain)
    finally:
        for h in (good, other, strided, nest):
            B.deco_orth_destroy(h)
        B.deco_destroy(plain)
        B.deco_destroy(server)


@gpu
def test_run_refusals():
    h = B.deco_orth_init(100, [(0, 10, 10)])
    x, out = torch.zeros(100, device="cuda"), torch.zeros(100, device="cuda", dtype=torch.bfloat16)
    try:
        for bad in ((x.half(), out, None), (x, out.float(), None), (x[:99], out, None), (x.double(), out, None),
                    (torch.zeros(200, device="cuda")[::2], out, None), (x, out, out), (x.cpu(), out, None)):
            with pytest.raises(ValueError):
                B.deco_orth_run(h, bad[0], bad[1], momentum=bad[2])
        lib = B.load()
        assert lib.deco_orth_run(h, x.data_ptr() + 2, B.DECO_F32, None, out.data_ptr(), None) == B.DECO_ERR_INVALID_ARG
        assert lib.deco_orth_run(h, x.data_ptr(), 5, None, out.data_ptr(), None) == B.DECO_ERR_INVALID_ARG
        assert lib.deco_orth_run(h, None, 0, None, out.data_ptr(), None) == B.DECO_ERR_INVALID_ARG
        assert lib.deco_orth_run(None, x.data_ptr(), 0, None, out.data_ptr(), None) == B.DECO_ERR_INVALID_ARG
    finally:
        B.deco_orth_destroy(h)
    empty = B.deco_orth_init(100, [])                               # no matrices: momentum alone
    try:
        m = torch.ones(100, device="cuda")
        B.deco_orth_run(empty, x, out, momentum=m)
        assert (m == 0).all() and (out == 0).all()
    finally:
        B.deco_orth_destroy(empty)


@pytest.mark.parametrize("kw", [dict(steps=17), dict(eps=-1.0), dict(momentum=1.0), dict(momentum=-0.1), dict(scale=3),
                                dict(scale=-1), dict(coef=(9.0, 0.0, 0.0)), dict(coef=(3.4445, -4.775, 9.0)),
                                dict(coef=(math.nan, 0.0, 0.0)), dict(eps=math.nan)])
def test_options_are_checked_on_the_host(kw):
    with pytest.raises(B.DecoError) as e:
        B.deco_orth_init(100, [(0, 10, 10)], **kw)
    assert e.value.status == B.DECO_ERR_INVALID_ARG


@pytest.mark.parametrize("mats", [[(0, 0, 5)], [(0, 5, 0)], [(1, 10, 10)], [(0, 5, 5), (24, 5, 5)], [(0, 2, 5, 4)],
                                  [(0, 4, 10, 20), (5, 4, 10, 20)], [(0, 4, 10, 20), (10, 3, 10, 21)],
                                  [(0, 4, 10, 20), (30, 1, 5)], [(2 ** 63, 1, 1)]])
def test_layouts_are_checked_on_the_host(mats):
    with pytest.raises(B.DecoError) as e:
        B.deco_orth_init(100, mats)
    assert e.value.status == B.DECO_ERR_INVALID_ARG


def test_init_without_a_device_fails_loudly():
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    with pytest.raises(B.DecoError) as e:
        B.deco_orth_init(100, [(0, 10, 10)])
    assert e.value.status == B.DECO_ERR_CUDA


def test_workload_matrices_cover_the_tensors():
    from paper_2507_17346_b200 import workloads as W
    wl = W.make_workload("resnet18", 0.25)
    mats = W.matrices(wl)
    assert len(mats) == 21 and all(r * c > 0 for _, r, c in mats)
    assert sum(r * c for _, r, c in mats) + sum(t.numel for t in wl.tensors if len(t.shape) == 1) == wl.d
    assert all(a[0] + a[1] * a[2] <= b[0] for a, b in zip(mats, mats[1:]))


@gpu
@pytest.mark.parametrize("name,scale", [("resnet18", 0.25), ("gpt2_small", 0.1), ("decoder_1b", 0.1)])
def test_workload_shapes(name, scale):
    """The workloads' own tensors (embeddings, convolutions, thin projections), vectors between them."""
    from paper_2507_17346_b200 import workloads as W
    wl = W.make_workload(name, scale)
    mats = W.matrices(wl)
    x = W.gradients_batched(wl, 0, W.entry_scales(wl, "cuda"))[0].contiguous()
    m = torch.zeros(wl.d, device="cuda")
    out = torch.zeros(wl.d, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(wl.d, mats, momentum=0.95)
    try:
        B.deco_orth_run(h, x, out, momentum=m)
        assert torch.equal(m, x.float())
        for at, r, c in mats:
            assert rel(out[at:at + r * c].view(r, c), exact(x[at:at + r * c].view(r, c))) < tol(r * c)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)


@gpu
def test_captured_in_a_graph():
    """A pass holds nothing that stream capture forbids: both kinds of matrices, fork and join included."""
    mats, d, x = flat_case([(64, 147), (300, 200), (520, 400)], 3, torch.float32, 9)
    out, again = (torch.zeros(d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    h = B.deco_orth_init(d, mats)
    try:
        B.deco_orth_run(h, x, out)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.deco_orth_run(h, x, again, stream=s)
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again)
    finally:
        B.deco_orth_destroy(h)


@gpu
def test_example_trains():
    """Loss, compressed exchange and orthogonalised update together: the loss falls most of the way from
    log(vocab) to the entropy rate of the tokens."""
    from paper_2507_17346_b200 import example_lm
    losses, model, chain = example_lm.train(steps=120, workers=3, vocab=256, width=64, hidden=128, batch=512)
    start, floor = math.log(256), chain.entropy_rate()
    assert abs(losses[0] - start) < 1.0
    assert losses[-1] < floor + 0.5 * (start - floor), (losses[0], losses[-1], floor)
    found, entropy = example_lm.alternatives(model, 7)
    assert len(found) == 5 and all(a[1] >= b[1] for a, b in zip(found, found[1:])) and entropy > 0


def test_tensor_memory_is_taken_before_dependents_may_start():
    """In every kernel that takes tensor memory, the allocation and a block barrier come before
    griddepcontrol.launch_dependents: a dependent that holds columns waits for this launch to end."""
    import os
    import re
    path = os.path.join(os.path.dirname(B.__file__), "csrc", "deco_orth.cu")
    kernels = re.split(r"^__global__", open(path).read(), flags=re.M)[1:]
    seen = 0
    for k in kernels:
        k = re.split(r"^}", k, flags=re.M)[0]
        if "tcgen05.alloc" not in k or "griddepcontrol.launch_dependents" not in k:
            continue
        seen += 1
        alloc, start = k.rindex("tcgen05.alloc"), k.index("griddepcontrol.launch_dependents")
        assert alloc < start and "__syncthreads()" in k[alloc:start]
    assert seen == 2


@gpu
def test_short_sides_alone_on_the_callers_stream():
    """Matrices of every cluster size and nothing else: their launches overlap on the caller's stream."""
    mats, d, x = flat_case([(64, 147), (64, 900), (1100, 30), (20, 4000), (100, 128), (200, 90), (120, 700), (1, 5000)],
                           3, torch.float32, 17)
    m = torch.zeros(d, device="cuda")
    out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(d, mats, momentum=0.9)
    try:
        for _ in range(3):
            B.deco_orth_run(h, x, out, momentum=m)
        for at, r, c in mats:
            assert rel(out[at:at + r * c].view(r, c), exact(m[at:at + r * c].view(r, c))) < tol(r * c)
        st = B.deco_orth_get_stats(h)
        assert st["device_status"] == 0 and st["groups"] == 0
    finally:
        B.deco_orth_destroy(h)


# ------------------------------------------------------- every way through the products on tiles

# short sides up to 128 whose entries no cluster holds (hi and lo of every operand), up to 256 (of P), above
GENERAL = [(100, 1300), (1301, 99), (128, 1040), (200, 333), (333, 201), (256, 1024), (300, 301), (301, 300), (520, 264),
           (640, 385), (768, 768), (1025, 520)]


def check_all(out, y, mats, scale=1.0):
    """Every matrix of `out` against the polynomial of `y`, the other entries against -9."""
    used = torch.zeros(len(out), dtype=torch.bool, device="cuda")
    for q in mats:
        pick = lambda t: torch.as_strided(t, (q[1], q[2]), (q[3] if len(q) > 3 else q[2], 1), q[0])  # noqa: B023, E731
        assert not pick(used).any()
        pick(used).fill_(True)
        assert rel(pick(out), scale * exact(pick(y))) < tol(q[1] * q[2]), q
    assert (out[~used] == -9).all()


@gpu
@pytest.mark.parametrize("tile_ctas", [1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap", [3, 8])
def test_one_cta_and_pairs_in_every_phase(tile_ctas, dtype, gap):
    """The three phases on tiles of one CTA and of a pair, for every precision, orientation and alignment."""
    mats, d, x = flat_case(GENERAL, gap, dtype, 23)
    out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(d, mats, tile_ctas=tile_ctas)
    try:
        B.deco_orth_run(h, x, out)
        check_all(out, x, mats)
        first = out.clone()
        B.deco_orth_run(h, x, out)
        assert torch.equal(out, first)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)


@gpu
@pytest.mark.parametrize("tile_ctas", [0, 1, 2])
@pytest.mark.parametrize("nesterov", [None, False, True])
@pytest.mark.parametrize("S,lead", [(1500, 10), (1504, 16)])
def test_strided_matrices_above_the_short_sides(S, lead, nesterov, tile_ctas):
    """Column ranges of one buffer of rows, wide and tall ones with rows apart, plain ones between; without
    momentum (nesterov None) and with."""
    at = lead + 310 * S
    mats = [(lead, 310, 600, S), (lead + 600, 300, 500, S), (lead + 1100, 310, 381, S), (at, 700, 300, 304),
            (at + 700 * 304, 270, 900, 901), (at + 700 * 304 + 270 * 901, 300, 200), (at + 700 * 304 + 270 * 901 + 60000, 140, 200, 208)]
    d = mats[-1][0] + 140 * 208 + 5
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn(d, generator=g, device="cuda")
    m = None if nesterov is None else torch.randn(d, generator=g, device="cuda")
    out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(d, mats, momentum=0.5, nesterov=bool(nesterov), tile_ctas=tile_ctas)
    try:
        y = x.double() if m is None else 0.5 * m.double() + x.double()
        B.deco_orth_run(h, x, out, momentum=m)
        if m is not None:
            assert ((m.double() - y).abs() <= (y.abs() + x.double().abs()) * 2.0 ** -23).all()
        check_all(out, 0.5 * y + x.double() if nesterov else y, mats)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)


@gpu
@pytest.mark.parametrize("rows,cols", [(70, 90), (100, 1300), (200, 300), (300, 400), (400, 300)])
def test_extreme_norms_zero_nan_and_infinity(rows, cols):
    """In one launch and through the general way, whose entries are divided by the norm in fp32 or in double."""
    x = make(rows, cols, "normal", 1)
    for f in (1e30, 1e-30, 3e37):
        assert rel(run_one(x * f, eps=1e-38), exact(x * f, eps=1e-38)) < tol(x.numel())
    assert rel(run_one(x * 1e-9), exact(x * 1e-9)) < tol(x.numel())  # eps takes part
    assert (run_one(torch.zeros_like(x)) == 0).all()
    for bad in (math.nan, math.inf, -math.inf):
        for where in ((3, 4), (rows - 1, cols - 1)):
            y = x.clone()
            y[where] = bad
            assert torch.isnan(run_one(y)).all()


@gpu
@pytest.mark.parametrize("tile_ctas", [0, 1, 2])
@pytest.mark.parametrize("delta", [0.01, 0.5])
@pytest.mark.parametrize("gap", [8, 13])
def test_server_update_of_larger_matrices(gap, delta, tile_ctas):
    """The parameters' rows in fp32, 16 bytes at a time and singly; products with every precision, on one CTA and
    on pairs; sparse (0.01) and dense (0.5) aggregates; short sides beside them.  Tolerance as in test_server_update."""
    shapes, n, lr, wd, mu, steps = [(64, 148), (300, 400), (520, 264), (200, 512), (100, 1300), (1040, 300)], 2, 0.02, 0.1, 0.9, 2
    mats, d, _ = flat_case(shapes, gap, torch.float32, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    params = (0.05 * torch.randn(d, generator=g, device="cuda")).contiguous()
    want = params.double().clone()
    ctx = B.deco_init(d, n, delta, 0, lr, lr_at_server=True, params=params)
    h = B.deco_orth_init(d, mats, momentum=mu, scale=B.DECO_ORTH_SCALE_SPECTRAL, tile_ctas=tile_ctas)
    m = torch.zeros(d, device="cuda")
    wm = torch.zeros(d, device="cuda", dtype=torch.float64)
    mu32, lr32, w32 = (float(torch.tensor(v)) for v in (mu, lr, 1.0 / n))
    decay = float(torch.tensor(1.0) - torch.tensor(lr) * torch.tensor(wd))
    used = torch.zeros(d, dtype=torch.bool, device="cuda")
    for at, r, c in mats:
        used[at:at + r * c] = True
    try:
        for t in range(steps):
            B.deco_ef_compress(ctx, torch.randn(n, d, generator=g, device="cuda"))
            B.deco_aggregate_stale(ctx)
            k, buf = B.deco_get_k(ctx), B.deco_get_buffers(ctx)
            pairs = B.view_i32(buf["msg"], (n, buf["k_cap"], 2))[:, :k]
            s = torch.zeros(d, device="cuda", dtype=torch.float64)
            for i in range(n):
                s.index_add_(0, pairs[i, :, 0].long(), pairs[i, :, 1].contiguous().view(torch.float32).double())
            B.deco_apply_update_orth(ctx, h, m, wd)
            wm = mu32 * wm + w32 * s
            step = torch.zeros(d, device="cuda", dtype=torch.float64)
            for at, r, c in mats:
                y = math.sqrt(max(1.0, r / c)) * exact(wm[at:at + r * c].view(r, c))
                step[at:at + r * c] = y.reshape(-1)
            want = want * decay - lr32 * torch.where(used, step, wm)
            err = params.double() - want
            for at, r, c in mats:
                e, y = err[at:at + r * c], step[at:at + r * c]
                assert e.norm() <= 2.9e-3 * lr32 * y.norm() * (t + 1) + 1e-6 * want.norm(), (r, c)
            assert err[~used].norm() <= 1e-6 * want.norm()
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)
        B.deco_destroy(ctx)


@gpu
@pytest.mark.parametrize("shapes", [[(2304, 768)] * 12 + [(768, 768)] * 12, [(2303, 769)] * 6 + [(769, 771)] * 7,
                                    [(2048, 2048), (256, 2048), (5632, 2048), (2048, 5632)],
                                    [(96, 2048)] * 60 + [(2048, 200)] * 40])
def test_many_large_matrices(shapes):
    """What a server update of a language model has: enough tiles for pairs in every phase by the library's own choice."""
    mats, d, x = flat_case(shapes, 0, torch.bfloat16, 29)
    out = torch.full((d,), -9.0, device="cuda", dtype=torch.bfloat16)
    h = B.deco_orth_init(d, mats)
    try:
        B.deco_orth_run(h, x, out)
        check_all(out, x, mats)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)


def test_tile_ctas_is_checked_on_the_host():
    with pytest.raises(B.DecoError) as e:
        B.deco_orth_init(100, [(0, 10, 10)], tile_ctas=3)
    assert e.value.status == B.DECO_ERR_INVALID_ARG


@gpu
def test_matrices_whose_offsets_pass_32_bits():
    """One with rows 2^25 entries apart, short- and long-sided ones behind 2^32 entries: against the polynomial."""
    S, lead = 2 ** 25 + 8, 3
    at = lead + 150 * S
    mats = [(lead, 150, 200, S), (at, 60, 130), (at + 60 * 130, 300, 200), (at + 60 * 130 + 300 * 200, 140, 190, 201)]
    d = mats[-1][0] + 140 * 201 + 5
    assert at > 2 ** 32
    x = torch.zeros(d, dtype=torch.bfloat16, device="cuda")
    out = torch.full((d,), -9.0, dtype=torch.bfloat16, device="cuda")
    pick = lambda t, q: torch.as_strided(t, (q[1], q[2]), (q[3] if len(q) > 3 else q[2], 1), q[0])  # noqa: E731
    for i, q in enumerate(mats):
        pick(x, q).copy_(make(q[1], q[2], "normal", 80 + i, torch.bfloat16))
    h = B.deco_orth_init(d, mats)
    try:
        B.deco_orth_run(h, x, out)
        assert B.deco_orth_get_stats(h)["device_status"] == 0
    finally:
        B.deco_orth_destroy(h)
    for q in mats:
        y = pick(x, q).clone()
        assert rel(pick(out, q), exact(y)) < tol(y.numel())
        pick(out, q).fill_(-9.0)
    for lo in range(0, d, 2 ** 30):
        assert (out[lo:lo + 2 ** 30] == -9).all()
