"""The verification where r is one or more: the last word with a weight, whatever the sums' order has made of the total.

Sharp distributions (logits of standard deviation 8), whose running sums in float64 are not exact: in some order of the additions an earlier word's
lies above the total by a rounding."""
import numpy as np
import pytest

from test_gpu_draft import Problem
from test_gpu_scan import _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,V,store", [(200, 32000, "f32"), (200, 32000, "bf16"), (60, 40003, "f32"), (60, 65536, "f32"), (60, 50021, "bf16"), (300, 700, "f32"),
                                       (65, 100003, "f32")])
def test_r_of_one_and_more(B, V, store):
    torch, _, types = _torch()
    p = Problem(B, 1, V, store, seed=V, lengths=True)
    r = np.random.default_rng(V + 1)
    z = 8 * r.standard_normal((B, 2, V)).astype(np.float32)
    z = np.exp(z - z.max(-1, keepdims=True))
    z /= z.sum(-1, keepdims=True)
    p.target = torch.from_numpy(z).to(types[store])
    p.draft = torch.from_numpy(np.ascontiguousarray(z[:, :1, ::-1])).to(types[store])
    above = np.array([1.0, 1.0, 1.0, np.nextafter(np.float32(1), np.float32(2)), 2.0, np.inf], np.float32)
    p.r = torch.from_numpy(above[np.arange(B) % len(above)])
    tokens, taken = p.run()
    target, draft = p.target.double().numpy(), p.draft.double().numpy()
    wrong = []
    for b in range(B):
        a = taken[b]
        w = target[b, a] - (draft[b, a] if a < p.n[b] else 0.0)
        last = np.flatnonzero((w if (w > 0).any() else target[b, a]) > 0)[-1]
        if tokens[b, a] != last:
            wrong.append((b, int(a), int(tokens[b, a]), int(last)))
    assert not wrong, (len(wrong), wrong[:4])
    for x, y in zip((tokens, taken), p.want()):
        assert np.array_equal(x, y)
