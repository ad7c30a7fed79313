"""One row in place: a single row has no distance to the next, so whatever its arguments say of it, the buffers are the same.  Refusals on the
host, with the library's launches going nowhere; the results on a device."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B
from paper_2507_17346_b200 import build
from tests.test_norm_host import P, invoke


def test_strides_of_one_row_are_not_compared():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no kernel could be launched")
    build.build()
    lib = B.load()
    for name, change in (("deco_layernorm", dict(y=P, y_stride=80)), ("deco_layernorm", dict(sum=P, sum_stride=80)),
                         ("deco_layernorm_grad", dict(dx=P, dx_stride=80))):
        assert invoke(lib, name, rows=2, **change) == B.DECO_ERR_INVALID_ARG
        assert invoke(lib, name, rows=1, **change) == B.DECO_ERR_CUDA            # nothing wrong but the missing device
        assert invoke(lib, name, rows=1, **{k: 63 if k.endswith("stride") else v for k, v in change.items()}) == B.DECO_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [50, 64, 9000])
def test_a_row_of_a_wider_buffer_in_place(cols, dtype):
    build.build()
    B.load()
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    new = lambda: torch.randn(4, cols + 32, generator=g, device="cuda").to(dtype)  # noqa: E731
    x, add, dy = new(), new(), new()
    mean, rstd = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")

    def run(x, add, y, total, dy, dx):
        """Norm with residual, the gradient of what it made, from rows [1, cols]."""
        B.deco_layernorm(x, None, None, y, mean=mean, rstd=rstd, add=add, total=total)
        B.deco_layernorm_grad(total, mean, rstd, None, dy, dx)
        return y.clone(), total.clone(), dx.clone()

    # (apart from one another: copies with the same distance between rows)
    part = lambda t: t.clone()[1:2, :cols]  # noqa: E731
    want = run(part(x), part(add), part(x), part(x), part(dy), part(dy))
    a, b, c = x.clone(), add.clone(), dy.clone()
    got = run(a[1:2, :cols], b[1:2, :cols], a[1:2, :cols], b[1:2, :cols], c[1:2, :cols], c[1:2, :cols])
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    for now, was in ((a, x), (b, add), (c, dy)):                   # and nothing beside the row is touched
        now[1, :cols] = was[1, :cols]
        assert torch.equal(now, was)
