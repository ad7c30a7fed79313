"""The default stream named explicitly: the workspace that a wrapper makes is that stream's, and no other stream is handed its bytes
while the call's kernels have yet to run."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    torch.cuda.set_device(0)


def norm_grad(stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, dy = (torch.randn(4000, 768, generator=g, device="cuda") for _ in range(2))
    mean, rstd = x.mean(1), (x.var(1, correction=0) + 1e-5).rsqrt()
    out = torch.empty_like(x), torch.empty(768, device="cuda"), torch.empty(768, device="cuda")
    return lambda: B.deco_layernorm_grad(x, mean, rstd, None, dy, out[0], dweight=out[1], dbias=out[2], stream=stream), out


def weight_grad(stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x, dy = torch.randn(4100, 500, generator=g, device="cuda"), torch.randn(4100, 700, generator=g, device="cuda")
    packed = B.packed8_empty(4100, 500)
    B.deco_pack8(x, packed)
    out = torch.empty(700, 500, device="cuda"), torch.empty(700, device="cuda")
    return lambda: B.deco_weight_grad8(dy, packed, out[0], db=out[1], stream=stream), out


@pytest.mark.parametrize("make", [norm_grad, weight_grad])
@pytest.mark.parametrize("default", [lambda: 0, lambda: 1, torch.cuda.default_stream, torch.cuda.current_stream])
def test_the_default_stream_by_name(monkeypatch, make, default):
    rooms, plain = [], B._workspace

    def workspace(*args):
        room = plain(*args)
        rooms.append((room[1], room[2]))                           # (its address: the tensor goes with the call)
        return room

    monkeypatch.setattr(B, "_workspace", workspace)
    run, out = make(None)
    run()
    want = [t.clone() for t in out]
    run, out = make(default())
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                                  # (the call's kernels wait behind it: some 10 ms)
    run()
    address, nbytes = rooms[-1]
    handed = []
    for _ in range(40):                                            # more than torch's pool has
        with torch.cuda.stream(torch.cuda.Stream()):
            other = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
            handed.append(other.data_ptr())
            del other
    torch.cuda.synchronize()
    assert not any(p < address + nbytes and address < p + nbytes for p in handed)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
