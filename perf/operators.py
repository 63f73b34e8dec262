"""The vocabulary's side of a training step, measured: the token embedding and its gradient, the output layer's cross entropy
without kept logits and its gradients, and the clipping of all gradients by their global norm.

Each case is one pass through one operator.  `own` False: the plain form, elementary torch operations in 32 bits, rounded once at
the end.  `own` True: the calls of include/echovocab.h and include/echoclip.h through the Python binding.

  embed_fwd   out[n] = scale * table[tokens[n]], zero where tokens[n] is no word
  embed_bwd   dtable[v] = scale * sum of dout[n] over tokens[n] == v;  "add": added to what is there, the gradient of an output
              layer that shares the table
  loss_fwd    loss[n] = lse[n] - (1 - s) z[n, label] - s mean_v z[n, v],  z = h W^T,  lse = log sum exp z;  both 0 without a label
  loss_step   the same, and dh, dW for given dloss
  clip        norm = sqrt(sum x^2) over all tensors;  x * min(1, max_norm / norm)
"""
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one decoder step of a batch of 64: where a launch's latency is the whole time
        {"name": "embed_step", "op": "embed_fwd", "N": 64, "V": 32000, "D": 512, "store": "f32", "out": "f32", "pad": 0.0},
        # a batch of 128 sentences of 100 words, some of them shorter
        {"name": "embed_batch_bf16", "op": "embed_fwd", "N": 12800, "V": 50021, "D": 1024, "store": "bf16", "out": "bf16", "pad": 0.3},
        # its gradient as the only one of the table (all of the table is written)
        {"name": "embed_grad_f32", "op": "embed_bwd", "N": 12800, "V": 32000, "D": 512, "store": "f32", "out": "f32", "pad": 0.4, "add": False},
        # added to the gradient of an output layer that shares the table; long sentences, wide odd rows
        {"name": "embed_grad_shared", "op": "embed_bwd", "N": 9601, "V": 50021, "D": 1020, "store": "bf16", "out": "bf16", "pad": 0.25, "add": True},
        # serving: the log-probability of one token, bound by one reading of W
        {"name": "score_one", "op": "loss_fwd", "N": 1, "V": 32000, "D": 1024, "store": "bf16", "out": "f32", "pad": 0.0, "smoothing": 0.0},
        # one decoder step of a batch of 64 scored
        {"name": "score_step_f32", "op": "loss_fwd", "N": 64, "V": 32000, "D": 512, "store": "f32", "out": "f32", "pad": 0.0, "smoothing": 0.0},
        # validation: losses of a batch of 128 sentences
        {"name": "score_batch_bf16", "op": "loss_fwd", "N": 12800, "V": 32000, "D": 512, "store": "bf16", "out": "f32", "pad": 0.4, "smoothing": 0.0},
        # training step of a small model in f32: 64 sentences of 50 words, an odd vocabulary, smoothed labels
        {"name": "train_f32", "op": "loss_step", "N": 3200, "V": 8003, "D": 512, "store": "f32", "out": "f32", "pad": 0.4, "smoothing": 0.1},
        # training step from bf16 storage, gradients in f32: 128 sentences of 50 words
        {"name": "train_bf16", "op": "loss_step", "N": 6400, "V": 32000, "D": 1024, "store": "bf16", "out": "f32", "pad": 0.45, "smoothing": 0.1},
        # a large vocabulary and wide rows, gradients in bf16
        {"name": "train_large_bf16", "op": "loss_step", "N": 8192, "V": 100003, "D": 2048, "store": "bf16", "out": "bf16", "pad": 0.0, "smoothing": 0.0},
        # the gradients of a small translation model
        {"name": "clip_small_f32", "op": "clip", "tensors": 18, "total": 1500000, "out": "f32", "max_norm": 1.0},
        # the gradients of a large one, many tensors of very different sizes
        {"name": "clip_large_bf16", "op": "clip", "tensors": 40, "total": 400000000, "out": "bf16", "max_norm": 5.0},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "loss_fwd", "loss_fwd", "loss_step", "loss_step", "clip"])
    if op == "clip":
        return {"op": op, "tensors": _log(rng, 1, 60), "total": _log(rng, 1000, 400000000), "out": rng.choice(["f32", "bf16"]), "max_norm": rng.choice([0.5, 1.0, 5.0])}
    c = {"op": op, "V": _log(rng, 500, 100003), "D": _log(rng, 60, 2048), "store": rng.choice(["f32", "bf16"]), "pad": rng.choice([0.0, 0.2, 0.45])}
    if rng.random() < 0.7:
        c["D"] = max(64, c["D"] // 8 * 8)          # most rows are whole groups of eight
    if op == "embed_fwd" or op == "embed_bwd":
        c["N"] = _log(rng, 1, 20000)
        c["out"] = rng.choice(["f32", "bf16"])
        if op == "embed_bwd":
            c["add"] = rng.random() < 0.5
        return c
    c["smoothing"] = rng.choice([0.0, 0.1])
    c["N"] = _log(rng, 1, 13000) if op == "loss_fwd" else _log(rng, 16, 13000)
    c["out"] = "f32" if op == "loss_fwd" or c["store"] == "f32" else rng.choice(["f32", "bf16"])
    most = 2 * 8192 * 100003 * 2048 // (1 if c["store"] == "bf16" else 6)
    c["N"] = max(1, min(c["N"], most // (2 * c["V"] * c["D"])))
    return c


def work(case):
    if case["op"] == "clip":
        b = 2 if case["out"] == "bf16" else 4
        return {"bytes": case["total"] * 2 * b, "flops": case["total"] * 3}
    N, V, D = case["N"], case["V"], case["D"]
    i, o = (2 if case["store"] == "bf16" else 4), (2 if case["out"] == "bf16" else 4)
    if case["op"] == "embed_fwd":
        return {"bytes": N * 4 + min(N, V) * D * i + N * D * o, "flops": N * D}
    if case["op"] == "embed_bwd":
        return {"bytes": N * 4 + N * D * o + (2 * min(N, V) if case["add"] else V) * D * 4, "flops": N * D}
    rows = int(N * (1 - case["pad"]))              # rows without a label take part in nothing
    if case["op"] == "loss_fwd":
        return {"bytes": (rows + V) * D * i + N * 12, "flops": 2 * rows * V * D}
    return {"bytes": (rows + V) * D * i + (N + V) * D * o + N * 16, "flops": 8 * rows * V * D}


def _sizes(case):
    """Sizes of the tensors of a model's gradients: a few large matrices, many small ones, each its share of `total`."""
    k, left, out = case["tensors"], case["total"], []
    for j in range(k - 1):
        n = max(1, left // (2 if j < 4 else 7) - 3 * j)
        n = min(n, left - (k - 1 - j))
        out.append(n)
        left -= n
    return out + [left]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "clip":
        t = TYPES[case["out"]]
        s["grads"] = [(torch.randn(n, device="cuda", generator=g) * (0.02 / (1 + j % 3))).to(t) for j, n in enumerate(_sizes(case))]
        s["clipped"] = [torch.empty_like(x) for x in s["grads"]]
        return s
    N, V, D = case["N"], case["V"], case["D"]
    store, out = TYPES[case["store"]], TYPES[case["out"]]
    # words by Zipf's law; the ends of short sentences hold no word
    words = torch.exp(torch.rand(N, device="cuda", generator=g) * torch.log(torch.tensor(V + 0.5, device="cuda"))).to(torch.int32) - 1
    words = words.clamp_(0, V - 1)
    if case["pad"]:
        length = 50
        short = torch.rand((N + length - 1) // length, device="cuda", generator=g) * 2 * case["pad"]
        place = torch.arange(N, device="cuda")
        words = torch.where((place % length + 1) > length * (1 - short[place // length]), torch.full_like(words, -1), words)
    s["words"] = words
    if case["op"] == "embed_fwd":
        s["table"] = (torch.randn(V, D, device="cuda", generator=g) / D ** 0.5).to(store)
        s["result"] = torch.empty(N, D, device="cuda", dtype=out)
        return s
    if case["op"] == "embed_bwd":
        s["dout"] = (torch.randn(N, D, device="cuda", generator=g) * 1e-3).to(out)
        s["dtable"] = torch.randn(V, D, device="cuda", generator=g) * 1e-3 if case["add"] else torch.empty(V, D, device="cuda")
        return s
    W = torch.randn(V, D, device="cuda", generator=g) / D ** 0.5
    h = 1.5 * torch.randn(N, D, device="cuda", generator=g)
    # the label's probability runs from one in the vocabulary to nearly one
    sure = torch.rand(N, 1, device="cuda", generator=g) * 14
    h += sure * W[words.clamp(min=0).long()]
    s["W"], s["h"] = W.to(store), h.to(store)
    if case["op"] == "loss_step":
        valid = (words >= 0).float()
        s["dloss"] = valid / valid.sum().clamp(min=1)
    return s


def _plain_clip(s):
    norm = sum((x.float().square().sum() for x in s["grads"]), torch.zeros((), device="cuda")).sqrt()
    factor = (s["max_norm"] / norm).clamp(max=1.0)
    return {"norm": norm.reshape(1), "clipped": [(x.float() * factor).to(x.dtype) for x in s["grads"]]}


def _plain_loss(s):
    V, eps = s["V"], s["smoothing"]
    h, W = s["h"].float(), s["W"].float()
    label = s["words"].long()
    valid = label >= 0
    at = label.clamp(min=0)[:, None]
    z = h @ W.t()
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    loss = (lse - (1 - eps) * z.gather(1, at))[:, 0] - eps * z.mean(1)
    none = torch.zeros_like(loss)
    result = {"loss": torch.where(valid, loss, none), "lse": torch.where(valid, lse[:, 0], none)}
    if s["op"] == "loss_fwd":
        return result
    dz = (z - lse).exp() - eps / V
    dz.scatter_add_(1, at, torch.full_like(at, -(1 - eps), dtype=torch.float32))
    dz *= torch.where(valid, s["dloss"], none)[:, None]
    out = TYPES[s["out"]]
    return result | {"dh": (dz @ W).to(out), "dW": (dz.t() @ h).to(out)}


def _plain(s):
    if s["op"] == "clip":
        return _plain_clip(s)
    if s["op"] in ("loss_fwd", "loss_step"):
        return _plain_loss(s)
    valid = (s["words"] >= 0)[:, None]
    at = s["words"].clamp(min=0).long()
    scale = s["D"] ** 0.5
    if s["op"] == "embed_fwd":
        rows = s["table"][at].float() * scale
        return (rows * valid).to(TYPES[s["out"]])
    rows = s["dout"].float() * scale * valid
    into = s["dtable"] if s["add"] else torch.zeros_like(s["dtable"])
    return into.index_add_(0, at, rows)


def _plan(s):
    """What a user's program keeps between steps: descriptor, results and workspace."""
    from paper_1805_08899_amd import binding as eb

    def bytes_(n):
        return torch.empty(max(int(n), 16), dtype=torch.uint8, device="cuda")

    p = {"eb": eb}
    if s["op"] == "clip":
        p["grads"] = eb.make_grads(s["grads"], s["clipped"])
        p["norm"] = torch.empty(1, device="cuda")
        p["ws"] = bytes_(eb.echo_grad_workspace_bytes(p["grads"], len(s["grads"])))
        return p
    N, D = s["N"], s["D"]
    p["desc"] = d = eb.make_vocab_desc(N, s["V"], D, s["store"], s["out"])
    if s["op"] == "embed_bwd":
        p["ws"] = bytes_(eb.echo_embed_bwd_workspace_bytes(d))
    elif s["op"] != "embed_fwd":
        p["loss"], p["lse"] = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        n = eb.echo_vocab_loss_fwd_workspace_bytes(d)
        if s["op"] == "loss_step":
            n = max(n, eb.echo_vocab_loss_bwd_workspace_bytes(d))
            p["dh"], p["dW"] = torch.empty_like(s["h"], dtype=TYPES[s["out"]]), torch.empty_like(s["W"], dtype=TYPES[s["out"]])
        p["ws"] = bytes_(n)
    return p


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    p = s["plan"]
    eb, st = p["eb"], torch.cuda.current_stream()
    if s["op"] == "clip":
        eb.check(eb.echo_grad_clip(p["grads"], len(s["grads"]), s["max_norm"], p["norm"], p["ws"], stream=st), "echo_grad_clip")
        return {"norm": p["norm"], "clipped": s["clipped"]}
    d, scale = p["desc"], s["D"] ** 0.5
    if s["op"] == "embed_fwd":
        eb.check(eb.echo_embed_fwd(d, s["words"], s["table"], scale, s["result"], stream=st), "echo_embed_fwd")
        return s["result"]
    if s["op"] == "embed_bwd":
        call, name = (eb.echo_embed_bwd_accumulate, "echo_embed_bwd_accumulate") if s["add"] else (eb.echo_embed_bwd, "echo_embed_bwd")
        eb.check(call(d, s["words"], s["dout"], scale, s["dtable"], p["ws"], stream=st), name)
        return s["dtable"]
    eb.check(eb.echo_vocab_loss_fwd(d, s["h"], s["W"], s["words"], s["smoothing"], p["loss"], p["lse"], p["ws"], stream=st), "echo_vocab_loss_fwd")
    if s["op"] == "loss_fwd":
        return {"loss": p["loss"], "lse": p["lse"]}
    eb.check(eb.echo_vocab_loss_bwd(d, s["dloss"], p["lse"], s["h"], s["W"], s["words"], s["smoothing"], p["dh"], p["dW"], p["ws"], stream=st),
             "echo_vocab_loss_bwd")
    return {"loss": p["loss"], "lse": p["lse"], "dh": p["dh"], "dW": p["dW"]}


def run(state):
    if own:
        return _own(state)
    return _plain(state)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "clip":
        total = torch.zeros((), device="cuda", dtype=f64)
        for x in s["grads"]:
            x = x.to(f64)
            total += (x * x).sum()
        norm = torch.sqrt(total)
        factor = torch.minimum(torch.ones_like(norm), case["max_norm"] / norm)
        return {"norm": norm.reshape(1), "clipped": [x.to(f64).mul_(factor) for x in s["grads"]]}
    words = s["words"].to(torch.int64)
    rows = torch.nonzero(words >= 0)[:, 0]
    label = words[rows]
    N, V, D = case["N"], case["V"], case["D"]
    if case["op"] == "embed_fwd":
        out = torch.zeros(N, D, device="cuda", dtype=f64)
        out[rows] = s["table"].to(f64)[label] * (float(D) ** 0.5)
        return out
    if case["op"] == "embed_bwd":
        out = s["dtable"].to(f64) if case["add"] else torch.zeros(V, D, device="cuda", dtype=f64)
        out.index_put_((label,), s["dout"].to(f64)[rows] * (float(D) ** 0.5), accumulate=True)
        return out
    eps = case["smoothing"]
    h, W = s["h"].to(f64), s["W"].to(f64)
    step = case["op"] == "loss_step"
    loss, lse = torch.zeros(N, device="cuda", dtype=f64), torch.zeros(N, device="cuda", dtype=f64)
    dh, dW = (torch.zeros_like(h), torch.zeros_like(W)) if step else (None, None)
    for a in range(0, N, 1024):
        z = torch.matmul(h[a:a + 1024], W.transpose(0, 1))
        here = rows[(rows >= a) & (rows < a + 1024)]
        lse[here] = torch.logsumexp(z, dim=1)[here - a]
        y = words[here]
        wanted = (1 - eps) * z[here - a, y] + eps * z[here - a].sum(dim=1) / V
        loss[here] = lse[here] - wanted
        if step:
            p = torch.softmax(z, dim=1)
            target = torch.zeros_like(p)
            target[here - a, y] = 1 - eps
            target[here - a] += eps / V
            up = torch.zeros(p.shape[0], 1, device="cuda", dtype=f64)
            up[here - a, 0] = s["dloss"].to(f64)[here]
            dz = (p - target) * up
            dh[a:a + 1024] = torch.matmul(dz, W)
            dW += torch.matmul(dz.transpose(0, 1).contiguous(), h[a:a + 1024])
    return {"loss": loss, "lse": lse, "dh": dh, "dW": dW} if step else {"loss": loss, "lse": lse}
