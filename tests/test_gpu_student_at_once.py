"""Two calls of the recurrence, the distillation and the verification at once, on streams of their own: all buffers are there and filled before the first one is
issued, nothing is waited for in between, and each call's results are those that it has by itself."""
import numpy as np
import pytest

import test_gpu_distill
import test_gpu_draft
import test_gpu_scan
from test_gpu_scan import Buffers, _torch

pytestmark = pytest.mark.gpu


class Scan:
    def __init__(self, p, torch, eb, types):
        t, (B, T, H), b = types[p.store], (p.B, p.T, p.H), Buffers(torch)
        dev = lambda x: None if x is None else x.cuda()
        G, dh, c0, dc, n = dev(p.G), dev(p.dh), dev(p.c0), dev(p.dc_last), None if p.n is None else torch.from_numpy(p.n).cuda()
        self.out = dict(h=b.of(t, B, T, H), c_last=b.of(torch.float32, B, H), dG=b.of(t, B, T, 3 * H), dc0=b.of(torch.float32, B, H))
        states, ws = b.bytes(eb.echo_scan_states_bytes(p.desc)), [b.bytes(max(16, f(p.desc))) for f in (eb.echo_scan_fwd_workspace_bytes, eb.echo_scan_bwd_workspace_bytes)]
        o, self.buffers = self.out, b

        def step(st):
            eb.check(eb.echo_scan_fwd(p.desc, G, c0, n, o["h"], o["c_last"], states, ws[0], stream=st))
            eb.check(eb.echo_scan_bwd(p.desc, dh, dc, G, n, states, o["dG"], o["dc0"], ws[1], stream=st))
        self.step = step


class Distill:
    def __init__(self, p, torch, eb, types):
        N, V, D, K, T, t, b = p.N, p.V, p.D, p.K, p.T, types[p.out], Buffers(torch)
        x, g = (p.h.cuda(), p.W.cuda(), torch.from_numpy(p.words).cuda(), p.logits.cuda()), p.dloss.cuda()
        self.out = dict(loss=b.of(torch.float32, N), lse=b.of(torch.float32, N), dh=b.of(t, N, D), dW=b.of(t, V, D))
        ws = [b.bytes(f(p.desc, K)) for f in (eb.echo_distill_fwd_workspace_bytes, eb.echo_distill_bwd_workspace_bytes)]
        o, self.buffers = self.out, b

        def step(st):
            eb.check(eb.echo_distill_fwd(p.desc, *x, K, T, o["loss"], o["lse"], ws[0], stream=st))
            eb.check(eb.echo_distill_bwd(p.desc, g, o["lse"], *x, K, T, o["dh"], o["dW"], ws[1], stream=st))
        self.step = step


class Draft:
    def __init__(self, p, torch, eb, types):
        b, d = Buffers(torch), eb.make_draft_desc(p.B, p.K, p.V, p.store)
        x = [torch.from_numpy(p.drafted).cuda(), torch.from_numpy(p.n).cuda(), p.draft.cuda(), p.target.cuda(), p.u.cuda(), p.r.cuda()]
        self.out = dict(tokens=b.of(torch.int32, p.B, p.K + 1), taken=b.of(torch.int32, p.B))
        ws, o, self.buffers = b.bytes(max(16, eb.echo_draft_verify_workspace_bytes(d))), self.out, b
        self.step = lambda st: eb.check(eb.echo_draft_verify(d, *x, o["tokens"], o["taken"], ws, stream=st))


scan, distill, draft = test_gpu_scan.Problem, test_gpu_distill.Problem, test_gpu_draft.Problem
PAIRS = {
    # chains of many blocks on both streams, each with more blocks than the chip holds by itself
    "chains": lambda: (Scan, scan(8, 900, 520, seed=50), scan(12, 700, 260, "bf16", True, "random", seed=51)),
    "a long chain and short sequences": lambda: (Scan, scan(1, 9000, 70, seed=52), scan(40, 50, 130, "bf16", False, "random", seed=53)),
    "chains and walks": lambda: (Scan, scan(4, 1500, 200, "bf16", seed=54), scan(64, 250, 256, reverse=True, lengths="random", seed=55)),
    "tiles and few rows": lambda: (Distill, distill(1500, 3000, 128, 20, "bf16", T=2.0, seed=56), distill(60, 3000, 64, 9, seed=57)),
    "tiles": lambda: (Distill, distill(900, 2000, 128, 20, "bf16", "bf16", seed=58), distill(700, 1500, 100, 9, T=1.5, seed=59)),
    "several blocks and one to a sequence": lambda: (Draft, draft(5, 3, 70001, seed=60), draft(90, 2, 9001, "bf16", seed=61)),
    "several blocks to a sequence": lambda: (Draft, draft(7, 2, 50021, "bf16", seed=62), draft(3, 4, 100003, seed=63)),
}


@pytest.mark.parametrize("pair", sorted(PAIRS))
def test_two_at_once(pair):
    torch, eb, types = _torch()
    make, *problems = PAIRS[pair]()
    runs = [make(p, torch, eb, types) for p in problems]
    streams = [torch.cuda.Stream() for _ in runs]
    want = []
    for r in runs:
        r.step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append({k: x.clone() for k, x in r.out.items()})
        for x in r.out.values():
            x.view(torch.uint8).fill_(0xFF)
    torch.cuda.synchronize()
    for _ in range(8):
        for r, st in zip(runs, streams):
            r.step(st)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        r.buffers.check()
        for k, x in r.out.items():
            assert torch.equal(x.contiguous().view(torch.uint8), w[k].contiguous().view(torch.uint8)), k
        assert all(bool(torch.isfinite(x.float()).all()) for k, x in r.out.items())
    for p, w in zip(problems, want):
        got = p.run()
        for k, x in zip(w, got if isinstance(got, tuple) else [got[k] for k in w]):
            assert np.array_equal(w[k].double().cpu().numpy(), x), k


def test_the_verification_on_another_stream():
    torch, eb, types = _torch()
    for p in (draft(3, 2, 60001, seed=64), draft(70, 2, 500, seed=65)):
        run, st = Draft(p, torch, eb, types), torch.cuda.Stream()
        torch.cuda.synchronize()
        run.step(st)
        torch.cuda.synchronize()
        for k, x in zip(("tokens", "taken"), p.want()):
            assert np.array_equal(run.out[k].cpu().numpy(), x), k
        run.buffers.check()
