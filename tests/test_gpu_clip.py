"""Global gradient norm and clipping against the float64 oracle.

Tolerances.  The norm is an fp64 sum rounded to fp32 once: 2^-24 of it (the fp64 roundings are below 2^-40 of it).  A clipped element
is one fp32 product with a factor that was rounded once (2^-24 each), rounded to its type: fp32 2 x 2^-24 together, bf16 2^-8 + 2 x 2^-24."""
import numpy as np
import pytest

from oracle import vocab_ref as vr

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    assert torch.cuda.is_available(), "needs the GPU"
    from paper_1805_08899_amd import binding as eb
    return torch, eb


def _tensors(torch, sizes, scale, seed, types=("f32", "bf16")):
    g = torch.Generator()
    g.manual_seed(seed)
    kinds = {"f32": torch.float32, "bf16": torch.bfloat16}
    return [(torch.randn(n, generator=g) * scale).to(kinds[types[i % len(types)]]).cuda() for i, n in enumerate(sizes)]


SETS = {
    "one element": [1],
    "odd": [1, 3, 5, 4095, 4096, 4097, 8191, 8192, 8193, 0, 12289],
    "empty": [0, 0],
    "empty among others": [0, 7, 0, 0, 100000, 0],
    "many": [(37 * i) % 5000 for i in range(250)],           # three launches' worth
    "exactly one table": [10 + i for i in range(96)],
    "large": [20000003, 1, 8388608, 5],
}


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("name", sorted(SETS))
def test_norm_and_clipping(name, in_place):
    torch, eb = _torch()
    print("clip", name, in_place, flush=True)
    xs = _tensors(torch, SETS[name], 0.1, len(name))
    host = [x.double().cpu().numpy() for x in xs]
    norm = vr.grad_norm(host)
    n, st = len(xs), torch.cuda.current_stream()
    for limit in (0.3 * norm + 1e-6, 3.0 * norm + 1.0):
        src = [x.clone() for x in xs]
        dst = src if in_place else [torch.full_like(x, float("nan")) for x in xs]
        grads = eb.make_grads(src, dst)
        got = torch.full((1,), float("nan"), device="cuda")
        ws = torch.full((eb.echo_grad_workspace_bytes(grads, n),), 0xFF, dtype=torch.uint8, device="cuda")
        eb.check(eb.echo_grad_norm(grads, n, got, ws, stream=st))
        first = got.clone()
        got.fill_(float("nan"))
        eb.check(eb.echo_grad_clip(grads, n, limit, got, ws, stream=st))
        torch.cuda.synchronize()
        assert torch.equal(first, got)
        assert abs(float(got) - norm) <= 2.0 ** -24 * 1.01 * norm
        limit = float(np.float32(limit))
        _, want = vr.grad_clip(host, limit)
        for x, d, w in zip(xs, dst, want):
            if norm <= limit:
                assert torch.equal(d, x), "nothing to clip"
                continue
            bound = (2.0 ** -8 if d.dtype == torch.bfloat16 else 0) + 2.02 * 2.0 ** -24
            assert (np.abs(d.double().cpu().numpy() - w) <= bound * np.abs(w)).all()
        if not in_place:
            assert all(torch.equal(a, b) for a, b in zip(src, xs)), "the gradients themselves are left alone"


@pytest.mark.parametrize("scale", [1e30, 1e-30])
def test_squares_neither_overflow_nor_vanish(scale):
    torch, eb = _torch()
    xs = _tensors(torch, [1000, 33], scale, 1, ("f32",))
    norm = vr.grad_norm([x.double().cpu().numpy() for x in xs])
    grads, got = eb.make_grads(xs), torch.empty(1, device="cuda")
    ws = torch.empty(eb.echo_grad_workspace_bytes(grads, 2), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_grad_clip(grads, 2, 1.0, got, ws, stream=torch.cuda.current_stream()))
    assert abs(float(got) - norm) <= 2.0 ** -23 * norm
    after = vr.grad_norm([x.double().cpu().numpy() for x in xs])
    assert abs(after - min(1.0, norm)) <= 1e-6 * min(1.0, norm)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_clips_nothing(bad):
    torch, eb = _torch()
    xs = _tensors(torch, [9000, 33], 1.0, 2)
    xs[1][7] = bad
    keep = [x.clone() for x in xs]
    grads, got = eb.make_grads(xs), torch.empty(1, device="cuda")
    ws = torch.empty(eb.echo_grad_workspace_bytes(grads, 2), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_grad_clip(grads, 2, 1.0, got, ws, stream=torch.cuda.current_stream()))
    assert not np.isfinite(float(got))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(xs, keep))


def test_no_limit():
    torch, eb = _torch()
    xs = _tensors(torch, [100], 1.0, 3)
    keep = xs[0].clone()
    grads, got = eb.make_grads(xs), torch.empty(1, device="cuda")
    ws = torch.empty(eb.echo_grad_workspace_bytes(grads, 1), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_grad_clip(grads, 1, float("inf"), got, ws, stream=torch.cuda.current_stream()))
    assert torch.equal(xs[0], keep) and float(got) > 0


def test_replayed_from_a_graph():
    """The graph holds the addresses: the array may be gone, the gradients new."""
    torch, eb = _torch()
    xs = _tensors(torch, [5000, 70000, 3], 1.0, 4)
    out = [torch.empty_like(x) for x in xs]
    got = torch.empty(1, device="cuda")
    ws = torch.empty(8192, dtype=torch.uint8, device="cuda")

    def clip():
        grads = eb.make_grads(xs, out)
        eb.check(eb.echo_grad_clip(grads, 3, 2.0, got, ws, stream=torch.cuda.current_stream()))

    clip()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip()
    for k in range(4):
        for x in xs:
            x.normal_(std=0.001 if k == 2 else 1.0)          # the third time there is nothing to clip
        clip()
        torch.cuda.synchronize()
        want = [got.clone()] + [x.clone() for x in out]
        for x in [got] + out:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([got] + out, want)), k
