"""The vocabulary loss bit for bit: its kernels are the distillation's too, and what is changed there must not change the labels' results.

tests/golden/vocab_loss_bits.txt holds the SHA-256 of loss, lse, dh and dW as the library gave them before it had a distillation, for inputs that are made with
integer arithmetic; `python tests/test_gpu_vocab_bits.py` prints the table of the library as it is."""
import hashlib
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
pytestmark = pytest.mark.gpu
GOLDEN = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "vocab_loss_bits.txt")

CASES = [
    # N, V, D, storage, gradients, smoothing: rows alone, in LDS, in groups; tiles of 128 and 256; dz as one plane of fp16, two, and three of bf16
    (1, 501, 64, "f32", "f32", 0.0), (7, 3000, 200, "bf16", "f32", 0.1), (16, 900, 1024, "f32", "f32", 0.0), (30, 1201, 96, "bf16", "bf16", 0.0),
    (64, 5000, 128, "f32", "f32", 0.1), (200, 4001, 256, "f32", "f32", 0.0), (300, 2000, 513, "bf16", "bf16", 0.0), (129, 700, 99, "f32", "f32", 0.1),
    (700, 1500, 260, "bf16", "f32", 0.1), (1500, 8003, 128, "f32", "f32", 0.0), (4300, 4000, 64, "bf16", "bf16", 0.1), (4300, 4000, 64, "bf16", "f32", 0.0),
    (4300, 4000, 64, "f32", "f32", 0.1),
]


def _numbers(n, seed, bits):
    """n whole numbers of -2^(bits - 1) .. 2^(bits - 1) - 1, by a multiplicative hash of their places."""
    x = np.arange(n, dtype=np.uint64) + np.uint64(seed << 40)
    for k in (0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB):
        x = (x ^ (x >> np.uint64(29))) * np.uint64(k)
    return (x >> np.uint64(64 - bits)).astype(np.int64) - (1 << (bits - 1))


def _sums(N, V, D, store, out, smoothing):
    import torch
    from paper_1805_08899_amd import binding as eb
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    bits = 22 if store == "f32" else 8
    matrix = lambda rows, seed, size: torch.from_numpy((_numbers(rows * D, seed, bits) * (size / 2 ** bits)).astype(np.float32).reshape(rows, D)).to(types[store]).cuda()
    h, W = matrix(N, 1, 4.0), matrix(V, 2, 1.0 / (1 << int(np.log2(D) // 2)))
    labels = np.abs(_numbers(N, 3, 30)) % (V + V // 8 + 1)       # some are none
    labels = torch.from_numpy(labels.astype(np.int32)).cuda()
    dloss = torch.from_numpy((_numbers(N, 4, 20) / 2.0 ** 18).astype(np.float32)).cuda()
    d, st = eb.make_vocab_desc(N, V, D, store, out), torch.cuda.current_stream()
    loss, lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    dh, dW = torch.empty(N, D, dtype=types[out], device="cuda"), torch.empty(V, D, dtype=types[out], device="cuda")
    ws = torch.empty(max(eb.echo_vocab_loss_fwd_workspace_bytes(d), eb.echo_vocab_loss_bwd_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    eb.check(eb.echo_vocab_loss_fwd(d, h, W, labels, smoothing, loss, lse, ws, stream=st))
    eb.check(eb.echo_vocab_loss_bwd(d, dloss, lse, h, W, labels, smoothing, dh, dW, ws, stream=st))
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(x.float()).all()) for x in (loss, lse, dh, dW))
    return [hashlib.sha256(x.view(torch.uint8).cpu().numpy().tobytes()).hexdigest()[:32] for x in (loss, lse, dh, dW)]


def _name(case):
    return "_".join(str(x) for x in case)


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_bits(case):
    with open(GOLDEN) as f:
        golden = {line.split()[0]: line.split()[1:] for line in f if line.strip() and not line.startswith("#")}
    assert _sums(*case) == golden[_name(case)]


if __name__ == "__main__":
    print("# N_V_D_storage_gradients_smoothing, and 32 digits of SHA-256 of loss, lse, dh, dW")
    for case in CASES:
        print(_name(case), *_sums(*case), flush=True)
