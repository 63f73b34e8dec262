"""Token embedding and its gradient against the float64 oracle.

Tolerances.  Forward: one product and one rounding, half a step of the type of the result (fp32 2^-24, bf16 2^-8 of the value), after
the product's own 2^-24.  Backward: an entry is a sum of c fp32 numbers, added in some fixed order, times the scale (and added to
what is there): at most c + 2 roundings of partial sums, each at most 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest

from oracle import vocab_ref as vr

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _torch():
    import torch
    assert torch.cuda.is_available(), "needs the GPU"
    from paper_1805_08899_amd import binding as eb
    return torch, eb, {"f32": torch.float32, "bf16": torch.bfloat16}


def _guarded(torch, n_bytes, guard=256):
    """A buffer of n_bytes between two zones that nothing may write; all of it starts as NaN bit patterns."""
    whole = torch.full((n_bytes + 2 * guard + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    inner = whole[guard:guard + n_bytes]

    def check():
        assert bool((whole[:guard] == 0xFF).all()) and bool((whole[guard + n_bytes:] == 0xFF).all()), "written outside its buffer"
    return inner, check


def _tokens(kind, N, V, seed):
    r = np.random.default_rng(seed)
    if kind == "one word":
        t = np.full(N, V - 1)
    elif kind == "none":
        t = np.where(r.random(N) < 0.5, -1, V)
    elif kind == "zipf":
        t = np.minimum(np.exp(r.random(N) * np.log(V + 0.5)).astype(np.int64) - 1, V - 1)
        t[r.random(N) < 0.2] = -1
        t[r.random(N) < 0.05] = V
        t[r.random(N) < 0.02] = -2 ** 31
        t[r.random(N) < 0.02] = 2 ** 31 - 1
    elif kind == "one class":                           # of the sort's blocks, to which words are dealt in turn
        t = r.integers(0, max(1, V // 1024), N) * 1024
    elif kind == "sorted":
        t = np.sort(r.integers(0, V, N))
    else:
        t = r.integers(0, V, N)
    return t.astype(np.int32)


CASES = [
    # N, V, D, table/in, out, tokens
    (1, 1, 1, "f32", "f32", "uniform"),
    (1, 5, 7, "bf16", "bf16", "uniform"),
    (33, 4, 9, "f32", "bf16", "zipf"),
    (31, 64, 4, "bf16", "f32", "zipf"),
    (32, 65, 12, "f32", "f32", "one word"),
    (33, 3, 12, "f32", "f32", "one word"),
    (100, 200, 260, "bf16", "bf16", "none"),
    (64, 32000, 512, "f32", "f32", "uniform"),
    (1000, 129, 100, "f32", "f32", "zipf"),
    (3200, 8003, 61, "bf16", "bf16", "zipf"),
    (6400, 1000, 516, "f32", "f32", "sorted"),
    (12800, 50021, 64, "bf16", "bf16", "zipf"),
    (5003, 700001, 8, "f32", "f32", "uniform"),        # more words than the sort's blocks can take 64 of
    (20000, 7, 36, "f32", "f32", "zipf"),               # runs of thousands
    (40000, 2, 8, "bf16", "f32", "uniform"),
    (16, 10, 2100, "f32", "f32", "uniform"),            # rows wider than a wave's four loads
    (70, 10, 4099, "bf16", "bf16", "zipf"),
    (9000, 50000, 20, "f32", "f32", "one class"),
    (3000, 3000000, 16, "bf16", "bf16", "one class"),
]
IDS = ["N%d_V%d_D%d_%s_%s_%s" % (c[:5] + (c[5].replace(" ", "_"),)) for c in CASES]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    torch, eb, types = _torch()
    N, V, D, ti, to, kind = case
    print("embed fwd", case, flush=True)
    r = np.random.default_rng(N + V)
    table = torch.from_numpy(r.standard_normal((V, D)).astype(np.float32)).to(types[ti])
    tokens = _tokens(kind, N, V, D)
    size = N * D * (4 if to == "f32" else 2)
    raw, check = _guarded(torch, size)
    out = raw.view(types[to]).view(N, D)
    scale = 1.7
    eb.check(eb.echo_embed_fwd(eb.make_vocab_desc(N, V, D, ti, to), torch.from_numpy(tokens).cuda(), table.cuda(), scale, out,
                               stream=torch.cuda.current_stream()))
    torch.cuda.synchronize()
    check()
    ref = vr.embed_forward(tokens, table.double().numpy(), float(np.float32(scale)))
    got = out.double().cpu().numpy()
    assert (np.abs(got - ref) <= (HALF[to] + 2.0 ** -24 * 1.01) * np.abs(ref)).all()


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case, add):
    torch, eb, types = _torch()
    N, V, D, _, to, kind = case
    print("embed bwd", case, add, flush=True)
    r = np.random.default_rng(N * 3 + V)
    dout = torch.from_numpy(r.standard_normal((N, D)).astype(np.float32)).to(types[to])
    tokens = _tokens(kind, N, V, D)
    desc = eb.make_vocab_desc(N, V, D, "f32", to)
    raw, check = _guarded(torch, V * D * 4)
    ws, check_ws = _guarded(torch, eb.echo_embed_bwd_workspace_bytes(desc))
    dtable = raw.view(torch.float32).view(V, D)
    old = r.standard_normal((V, D)).astype(np.float32)
    call = eb.echo_embed_bwd_accumulate if add else eb.echo_embed_bwd
    results = []
    for _ in range(2):                                  # the second run finds what the first left in the workspace
        if add:
            dtable.copy_(torch.from_numpy(old))
        else:
            dtable.fill_(float("nan"))
        eb.check(call(desc, torch.from_numpy(tokens).cuda(), dout.cuda(), -0.3, dtable, ws, stream=torch.cuda.current_stream()))
        torch.cuda.synchronize()
        results.append(dtable.cpu().numpy())
    check()
    check_ws()
    assert np.array_equal(results[0], results[1]), "bit-identical from run to run"
    ref, size = vr.embed_backward(tokens, dout.double().numpy(), float(np.float32(-0.3)), V)
    count = np.zeros((V, 1))
    np.add.at(count, tokens[(tokens >= 0) & (tokens < V)], 1)
    if add:
        ref, size = ref + old, size + np.abs(old)
        untouched = count[:, 0] == 0
        assert np.array_equal(results[0][untouched], old[untouched])
    bound = (count + 2) * 2.0 ** -24 * 1.01 * size
    assert (np.abs(results[0] - ref) <= bound).all()


def test_offsets_past_32_bits():
    """Table and gradient of more than 2^32 bytes: the last word's row."""
    torch, eb, types = _torch()
    N, V, D = 3, 1200000, 1024
    tokens = torch.tensor([V - 1, 0, V - 1], dtype=torch.int32).cuda()
    table = torch.zeros(V, D, device="cuda")
    table[V - 1] = 2.0
    table[0] = 3.0
    out = torch.empty(N, D, device="cuda")
    desc = eb.make_vocab_desc(N, V, D)
    st = torch.cuda.current_stream()
    eb.check(eb.echo_embed_fwd(desc, tokens, table, 1.0, out, stream=st))
    assert bool((out == torch.tensor([2.0, 3.0, 2.0], device="cuda")[:, None]).all())
    ws = torch.empty(eb.echo_embed_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_embed_bwd(desc, tokens, out, 1.0, table, ws, stream=st))
    assert bool((table[V - 1] == 4.0).all()) and bool((table[0] == 3.0).all()) and not bool(table[1:V - 1].any())


def test_replayed_from_a_graph_and_on_another_stream():
    torch, eb, types = _torch()
    N, V, D = 500, 300, 64
    desc = eb.make_vocab_desc(N, V, D)
    table, dout = torch.randn(V, D, device="cuda"), torch.randn(N, D, device="cuda")
    tokens = torch.randint(-1, V, (N,), device="cuda").int()
    out, dtable = torch.empty(N, D, device="cuda"), torch.empty(V, D, device="cuda")
    ws = torch.empty(eb.echo_embed_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def both():
        st = torch.cuda.current_stream()
        eb.check(eb.echo_embed_fwd(desc, tokens, table, 2.0, out, stream=st))
        eb.check(eb.echo_embed_bwd(desc, tokens, dout, 2.0, dtable, ws, stream=st))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        tokens.copy_(torch.randint(-1, V, (N,), device="cuda"))
        dout.normal_()
        both()
        torch.cuda.synchronize()
        want = out.clone(), dtable.clone()
        out.fill_(float("nan"))
        dtable.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(dtable, want[1]), k
