"""f32 storage within the limits that include/echovocab.h names: operands from 2^-110 on are exact as three bf16 numbers, and nothing overflows below 2^104 while
gradients carry their factor of 2^24.  Tolerances: test_gpu_vocab_loss.py."""
import pytest

from test_gpu_vocab_loss import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power,dloss", [(90, 0), (-90, 0), (0, 92), (0, -80), (60, 30), (-60, -30)])
@pytest.mark.parametrize("N,V,D", [(12, 300, 64), (300, 900, 136), (900, 2003, 129), (1500, 6000, 136)])
def test_f32_operands_and_dloss_of_any_size(N, V, D, power, dloss):
    """h up, W down by a power of two leave the logits as they are."""
    p = Problem(N, V, D, "f32", "f32", 0.1, seed=N)
    p.h, p.W, p.dloss = p.h * 2.0 ** power, p.W * 2.0 ** -power, p.dloss * 2.0 ** dloss
    p.check(p.run())
