"""What the built library says of the kernels at the vocabulary's ends and of the clipping: none keeps registers in memory."""
import re

import pytest

from test_built_kernels import _kernels

KERNELS = ["k_embed_fwd", "k_embed_sort", "k_embed_sum", "k_embed_join", "k_vocab_rows", "k_vocab_largest", "k_vocab_pack", "k_vocab_logits",
           "k_vocab_few_alone", "k_vocab_few_shared", "k_vocab_few_finish", "k_vocab_loss_finish", "k_vocab_grads", "k_vocab_dw_finish",
           "k_vocab_dh_finish", "k_grad_norm", "k_grad_norm_finish", "k_grad_scale"]


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_instance_spills(kernel, tmp_path):
    found = {n: v for n, v in _kernels(tmp_path).items() if re.search(r"\d" + kernel + r"[IE]", n)}
    assert found, "no such kernel in the library"
    assert not {n: v for n, v in found.items() if v != (0, 0)}
