"""The longest sequence that the recurrence takes, 2^24 steps in 131072 chunks, against the same one in two calls with the state handed over between them.

Both go through the same maps; at the border a state is rounded once more, by u = 2^-24 of numbers below 4 (|c0| and |g| are), and what is stored in bf16 may fall on
the other side of a rounding: one step of bf16, 2^-7 of the value, and 1e-6 besides."""
import pytest

from test_gpu_scan import _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reverse", [False, True])
def test_the_longest_sequence(reverse):
    torch, eb, _ = _torch()
    T, H, st = 1 << 24, 16, torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(3)
    G = torch.empty(1, T, 3 * H, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    G[:, :, :H] += 3
    dh = torch.empty(1, T, H, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    c0, dc = torch.randn(1, H, device="cuda", generator=g).clamp(-3, 3), torch.randn(1, H, device="cuda", generator=g)

    def run(G, dh, c0, dc):
        n = G.shape[1]
        d = eb.make_scan_desc(1, n, H, "bf16", reverse)
        h, dG = torch.empty(1, n, H, dtype=torch.bfloat16, device="cuda"), torch.empty_like(G)
        c, dc0 = torch.empty(1, H, device="cuda"), torch.empty(1, H, device="cuda")
        states = torch.empty(eb.echo_scan_states_bytes(d), dtype=torch.uint8, device="cuda")
        ws = torch.empty(max(eb.echo_scan_fwd_workspace_bytes(d), eb.echo_scan_bwd_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        eb.check(eb.echo_scan_fwd(d, G, c0, None, h, c, states, ws, stream=st))

        def back(dc):
            eb.check(eb.echo_scan_bwd(d, dh, dc, G, None, states, dG, dc0, ws, stream=st))
            torch.cuda.synchronize()
            return dG, dc0
        return h, c, back
    h, c, back = run(G, dh, c0, dc)
    dG, dc0 = back(dc)
    first, second = (slice(T // 2, T), slice(0, T // 2)) if reverse else (slice(0, T // 2), slice(T // 2, T))
    cut = lambda x, where: x[:, where].contiguous()
    h1, c1, back1 = run(cut(G, first), cut(dh, first), c0, dc)
    h2, c2, back2 = run(cut(G, second), cut(dh, second), c1, dc)
    dG2, middle = back2(dc)
    dG1, dc0_halves = back1(middle)
    near = lambda a, b: bool(((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-6).all())
    assert near(h[:, first], h1) and near(h[:, second], h2) and near(c, c2)
    assert near(dG[:, first], dG1) and near(dG[:, second], dG2) and near(dc0, dc0_halves)
    assert bool((h[:, first] == h1).float().mean() > 0.999) and bool((dG[:, second] == dG2).float().mean() > 0.999)
