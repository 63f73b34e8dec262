"""Clipping at the ends of fp32's range.  Tolerance: as in test_gpu_clip.py, a factor rounded once and one product, 2^-24 each (bf16: 2^-8 more);
half a place of the smallest number, 2^-150 (bf16: 2^-134), where a result is that small."""
import numpy as np
import pytest

from oracle import vocab_ref as vr
from test_gpu_clip import _torch

pytestmark = pytest.mark.gpu


def _clip(torch, eb, xs, max_norm):
    grads, norm, other = eb.make_grads(xs), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(eb.echo_grad_workspace_bytes(grads, len(xs)), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_grad_norm(grads, len(xs), other, ws, stream=torch.cuda.current_stream()))
    eb.check(eb.echo_grad_clip(grads, len(xs), max_norm, norm, ws, stream=torch.cuda.current_stream()))
    assert torch.equal(norm, other)
    return float(norm)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, 3e38])
def test_a_norm_past_the_largest_number_reads_infinity_and_clips_nothing(type_, max_norm):
    """Finite gradients: four of 3e38 have a norm of 6e38.  What `norm` says is what happened."""
    torch, eb = _torch()
    xs = [torch.full((n,), 3e38, device="cuda").to(torch.float32 if type_ == "f32" else torch.bfloat16) for n in (1, 3)]
    xs += [torch.randn(9001, device="cuda")]
    keep = [x.clone() for x in xs]
    assert _clip(torch, eb, xs, max_norm) == np.inf
    assert all(torch.equal(a, b) for a, b in zip(xs, keep))


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e30, 5.0, 1.0, 1e-20, 1e-30, 2e-38, 1e-42])
@pytest.mark.parametrize("norm", [3.3e38, 1e38, 1e30, 1e-25])
def test_factors_too_small_for_fp32(norm, max_norm, type_):
    """From 1.0 / 8.5e37 on a factor is no normal number of fp32."""
    torch, eb = _torch()
    r = np.random.default_rng(3)
    xs = [r.standard_normal(n) for n in (1, 33, 4096, 9001)]
    size = np.sqrt(sum((x ** 2).sum() for x in xs))
    xs = [torch.from_numpy((x * (norm / size)).astype(np.float32)).to(torch.float32 if type_ == "f32" else torch.bfloat16).cuda() for x in xs]
    host = [x.double().cpu().numpy() for x in xs]
    max_norm = float(np.float32(max_norm))
    true, want = vr.grad_clip(host, max_norm)
    assert abs(_clip(torch, eb, xs, max_norm) - true) <= 1.01 * 2.0 ** -24 * true
    for x, w, h in zip(xs, want, host):
        got = x.double().cpu().numpy()
        if true <= max_norm:
            assert np.array_equal(got, h)
            continue
        half, least = (2.0 ** -8, 2.0 ** -134) if type_ == "bf16" else (0.0, 0.0)
        assert (np.abs(got - w) <= (half + 2.02 * 2.0 ** -24) * np.abs(w) + least + 2.0 ** -150).all()
