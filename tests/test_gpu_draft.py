"""The verification of drafted words against the float64 oracle: words are equal.

The sums differ from the oracle's in their order, by 2^-53 of the sum per addition; a random r comes within that of a border with a probability of
about 1e-11 per sequence.  Borders that are meant to be met have weights whose sums are exact in any order."""
import numpy as np
import pytest

from oracle import student_ref as sr
from test_gpu_scan import Buffers, _torch

pytestmark = pytest.mark.gpu


class Problem:
    def __init__(self, B, K, V, store="f32", seed=0, lengths=True, spread=0.7):
        torch, eb, types = _torch()
        self.B, self.K, self.V, self.store = B, K, V, store
        r = np.random.default_rng(seed)
        soft = lambda z: np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)
        z = 3 * r.standard_normal((B, K + 1, V))
        q = soft(z[:, :K] + spread * r.standard_normal((B, K, V)))
        to = lambda x: torch.from_numpy(x.astype(np.float32))
        self.target, self.draft = to(soft(z)).to(types[store]), to(q).to(types[store])
        self.drafted = (q.cumsum(-1) < r.random((B, K, 1))).sum(-1).clip(0, V - 1).astype(np.int32)
        self.n = r.integers(0, K + 1, B).astype(np.int32) if lengths else None
        self.u, self.r = to(r.random((B, K))), to(r.random(B))

    def run(self, stream=None):
        torch, eb, _ = _torch()
        b, d = Buffers(torch), eb.make_draft_desc(self.B, self.K, self.V, self.store)
        dev = lambda x: torch.from_numpy(x).cuda()
        tokens, taken = b.of(torch.int32, self.B, self.K + 1), b.of(torch.int32, self.B)
        size = eb.echo_draft_verify_workspace_bytes(d)
        eb.check(eb.echo_draft_verify(d, dev(self.drafted), None if self.n is None else dev(self.n), self.draft.cuda(), self.target.cuda(), self.u.cuda(),
                                      self.r.cuda(), tokens, taken, b.bytes(size) if size else None, stream=stream or torch.cuda.current_stream()))
        torch.cuda.synchronize()
        b.check()
        return tokens.cpu().numpy(), taken.cpu().numpy()

    def want(self):
        return sr.draft_verify(self.drafted, self.n, self.draft.double().numpy(), self.target.double().numpy(), self.u.numpy(), self.r.numpy())

    def check(self):
        got, want = self.run(), self.want()
        for x, y in zip(got, want):
            assert np.array_equal(x, y), np.argwhere(x != y)[:4]
        return got


@pytest.mark.parametrize("B,K,V,store", [(1, 1, 1, "f32"), (2, 3, 2, "bf16"), (3, 2, 5, "f32"), (7, 4, 63, "bf16"), (5, 8, 64, "f32"), (4, 5, 65, "f32"),
                                         (9, 3, 1023, "bf16"), (6, 7, 4097, "f32"), (1, 4, 32000, "f32"), (3, 65, 130, "bf16"), (2, 2, 100003, "f32"),
                                         (1, 3, 50021, "bf16"), (300, 1, 777, "f32"), (1, 130, 70, "f32"), (1, 1, 262147, "bf16"), (5, 2, 8193, "bf16")])
@pytest.mark.parametrize("lengths", [True, False])
def test_against_the_oracle(B, K, V, store, lengths):
    for seed in range(3):
        Problem(B, K, V, store, seed + V, lengths, spread=(0.7, 0.0, 3.0)[seed]).check()


@pytest.mark.parametrize("B,V,store", [(70, 65537, "f32"), (64, 65537, "bf16"), (3, 65536, "f32"), (65, 40001, "bf16"), (2, 39999, "f32"), (1, 131073, "f32")])
def test_where_segments_and_blocks_change(B, V, store):
    p = Problem(B, 1, V, store, seed=B, lengths=True)
    p.check()
    p.target[:, :] = 0                                       # nothing is left of p, nor of p behind q
    p.target[::2, :, V - 1] = 0.5                            # but for the last word of every other sequence
    p.draft[:, :, V - 1] = 0.75
    p.u[:] = 0.9
    p.check()


def test_all_kinds_of_endings_occur():
    p = Problem(300, 4, 200, seed=5)
    tokens, taken = p.check()
    assert {0, 1, 2, 3, 4} == set(taken.tolist()) and (taken < p.n).any() and (taken == p.n).any()


@pytest.mark.parametrize("V", [8, 512, 4096, 40000])
@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_borders(V, store):
    """Weights of 2^-k and none, r at every border and one step of fp32 to both sides: a word is drawn from its border on."""
    torch, _, types = _torch()
    places = np.unique(np.linspace(0, V - 1, 8).astype(int))
    w = np.zeros(V, np.float32)
    w[places] = 1.0 / 8
    border = np.arange(9, dtype=np.float32) / len(places)
    r = np.concatenate([border, np.nextafter(border, np.float32(0)), np.nextafter(border, np.float32(2)), [-1.0, np.nan, np.inf, -np.inf]]).astype(np.float32)
    p = Problem(len(r), 1, V, store, seed=6, lengths=False)
    p.target[:] = torch.from_numpy(w).to(types[store])
    p.n, p.r = np.zeros(len(r), np.int32), torch.from_numpy(r)
    p.draft[:] = float("nan")                                # not read
    p.drafted[:] = -7
    tokens, taken = p.check()
    assert (taken == 0).all() and (tokens[:, 1] == -1).all() and set(tokens[:, 0]) == set(places)
    assert tokens[0, 0] == places[0] and tokens[1, 0] == places[1] and tokens[len(places), 0] == places[-1]


@pytest.mark.parametrize("V", [70, 5000])
def test_what_is_no_weight(V):
    torch, _, _ = _torch()
    p = Problem(6, 2, V, seed=7, lengths=False)
    p.u[:] = 2.0                                            # u q < p hardly ever
    p.target[0, 0, 3:] = float("nan")
    p.target[1, 0, ::2] = float("inf")
    p.target[2, 0, 1:] = -1.0
    p.draft[3, 0, ::2] = float("nan")
    p.draft[4, 0] = p.target[4, 0]                          # nothing is left: the target itself
    p.draft[5, 0, 1::2] = -float("inf")
    p.check()
    p.target[:, :] = 0
    tokens, taken = p.check()
    # u q < 0 holds where q is minus infinity: for the last sequence's word, if its number is odd
    odd = int(p.drafted[5, 0]) % 2
    assert (tokens[:5] == -1).all() and taken.tolist() == [0, 0, 0, 0, 0, odd] and (tokens[5, odd:] == -1).all()


def test_drafted_words_that_are_none():
    p = Problem(5, 3, 100, seed=8, lengths=False)
    p.u[:] = 0.0
    p.drafted[0, 0], p.drafted[1, 1], p.drafted[2, 2], p.drafted[3, 0] = -1, 100, 2 ** 31 - 1, -2 ** 31
    _, taken = p.check()
    assert taken.tolist() == [0, 1, 2, 0, 3]


def test_lengths_outside_their_range_and_words_behind_them():
    torch, _, _ = _torch()
    p = Problem(4, 3, 50, seed=9, lengths=False)
    p.n = np.array([-5, 2 ** 31 - 1, 1, -2 ** 31], np.int32)
    p.draft[2, 1:], p.target[2, 2:], p.u[2, 1:] = float("nan"), float("nan"), float("nan")
    p.drafted[2, 1:] = 10 ** 9
    p.check()


def test_NaN_at_a_drafted_word():
    p = Problem(3, 2, 40, seed=10, lengths=False)
    p.u[:] = 0.0
    p.u[0, 1] = float("nan")
    p.target[1, 0, p.drafted[1, 0]] = float("nan")
    p.draft[2, 1, p.drafted[2, 1]] = float("nan")
    _, taken = p.check()
    assert taken.tolist() == [1, 0, 1]


@pytest.mark.parametrize("B,V", [(2, 600), (3, 100003)])
def test_captured_and_replayed(B, V):
    torch, eb, _ = _torch()
    K = 3
    p = Problem(B, K, V, seed=11)
    d = eb.make_draft_desc(B, K, V)
    x = [torch.from_numpy(p.drafted).cuda(), torch.from_numpy(p.n).cuda(), p.draft.cuda(), p.target.cuda(), p.u.cuda(), p.r.cuda()]
    tokens, taken = torch.empty(B, K + 1, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, eb.echo_draft_verify_workspace_bytes(d)), dtype=torch.uint8, device="cuda")

    def step():
        eb.check(eb.echo_draft_verify(d, *x, tokens, taken, ws, stream=torch.cuda.current_stream()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(5):
        x[4].uniform_()
        x[5].uniform_()
        step()
        torch.cuda.synchronize()
        want = tokens.clone(), taken.clone()
        tokens.fill_(-9), taken.fill_(-9), ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(taken, want[1])


def test_offsets_past_32_bits():
    """The last sequences of 2^31.3 probabilities against the same ones by themselves."""
    torch, eb, _ = _torch()
    B, K, V = 24, 7, 14000000
    d = eb.make_draft_desc(B, K, V, "bf16")
    target = torch.rand(B, K + 1, V, dtype=torch.bfloat16, device="cuda")
    draft = target[:, :K].contiguous()
    draft[:, :, ::3] *= 0.25
    drafted = torch.randint(0, V, (B, K), device="cuda").int()
    u, r = torch.rand(B, K, device="cuda"), torch.rand(B, device="cuda")
    st = torch.cuda.current_stream()
    out = []
    for first in (0, B - 1):
        n = B - first
        d = eb.make_draft_desc(n, K, V, "bf16")
        tokens, taken = torch.empty(n, K + 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        ws = torch.empty(max(16, eb.echo_draft_verify_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        args = [x[first:].clone() for x in (drafted, draft, target, u, r)]
        eb.check(eb.echo_draft_verify(d, args[0], None, *args[1:], tokens, taken, ws, stream=st))
        out.append((tokens[-1].clone(), taken[-1].clone()))
        del args
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    a = int(out[0][1])
    p, q = target[-1, a].double(), draft[-1, a].double() if a < K else torch.zeros((), device="cuda")
    w = (p - q).clamp(min=0)
    w = (w if bool((w > 0).any()) else p).cumsum(0)
    assert int(out[0][0][a]) == int((w <= r[-1].double() * w[-1]).sum())
