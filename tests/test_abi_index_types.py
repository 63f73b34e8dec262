"""Tokens, labels and key lengths are 32-bit integers: a tensor of another type, or of fewer numbers than the call reads, is refused by both
forms of the calls (the builtin ones and the ctypes ones), without a GPU."""
import importlib.util

import pytest

from paper_1805_08899_amd import binding as eb

A = 0x10000  # a fake, aligned, never dereferenced device address
N, V, D = 6, 7, 8


def _ctypes_form():
    """The module's own functions, before the builtin ones stand in their place."""
    spec = importlib.util.spec_from_file_location("paper_1805_08899_amd.binding_ctypes_form", eb.__file__)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module._install_native_calls = lambda L: None
    return module


FORMS = {"builtin": lambda: eb, "ctypes": _ctypes_form}


def _calls(m, x):
    """Every call with an index, each of which stops at a null pointer behind it if x is taken (echo_attn_bwd_static without a GPU: at its scratch)."""
    d, a = m.make_vocab_desc(N, V, D), m.make_desc(N, 1, 4, 8, 8)
    big = 1 << 50
    return {
        "embed_fwd": lambda: m.echo_embed_fwd(d, x, A, 1.0, None),
        "embed_bwd": lambda: m.echo_embed_bwd(d, x, A, 1.0, None, A, big),
        "embed_bwd_accumulate": lambda: m.echo_embed_bwd_accumulate(d, x, A, 1.0, None, A, big),
        "vocab_loss_fwd": lambda: m.echo_vocab_loss_fwd(d, A, A, x, 0.0, A, None, A, big),
        "vocab_loss_bwd": lambda: m.echo_vocab_loss_bwd(d, A, A, A, A, x, 0.0, None, None, A, big),
        "attn_fwd": lambda: m.echo_attn_fwd(a, A, A, A, A, x, A, None, A, big),
        "attn_bwd": lambda: m.echo_attn_bwd(a, A, A, A, A, A, A, x, A, A, A, None, A, big),
        "attn_bwd_static": lambda: m.echo_attn_bwd_static(a, A, A, A, A, A, A, x, A, A, A, None),
        "attn_bwd_accumulate": lambda: m.echo_attn_bwd_accumulate(a, A, A, A, A, A, A, x, A, A, A, None, A, big),
        "attn_step_fwd": lambda: m.echo_attn_step_fwd(a, A, A, A, A, x, A, None),
        "attn_step_bwd": lambda: m.echo_attn_step_bwd(a, A, A, A, A, A, A, x, A, A, A, None),
        "attn_step_bwd_query": lambda: m.echo_attn_step_bwd_query(a, 0, 1, A, A, A, A, A, A, x, A, None),
        "attn_steps_bwd_keys": lambda: m.echo_attn_steps_bwd_keys(a, A, A, A, A, A, x, A, A, A, None, A, big),
        "attn_fwd_stash": lambda: m.echo_attn_fwd_stash(a, A, A, A, A, x, A, A, None, A, big),
        "attn_bwd_stash": lambda: m.echo_attn_bwd_stash(a, A, A, A, A, A, x, A, A, A, None, A, big),
    }


@pytest.mark.parametrize("form", sorted(FORMS))
def test_index_tensors(form):
    import torch
    m = FORMS[form]()

    class Own(torch.Tensor):
        pass

    class Address:
        def is_contiguous(self):
            return True

        def data_ptr(self):
            return A

    good = [Address(), torch.zeros(N, dtype=torch.int32), torch.zeros(2, N, dtype=torch.int32), torch.zeros(N, dtype=torch.int32).as_subclass(Own), A]
    bad = [torch.zeros(N, dtype=t) for t in (torch.int64, torch.int16, torch.uint8, torch.float32)]
    bad += [torch.zeros(N, dtype=torch.int64).as_subclass(Own), torch.zeros(N - 1, dtype=torch.int32), torch.zeros(0, dtype=torch.int32),
            torch.zeros(N - 1, dtype=torch.int32).as_subclass(Own), torch.zeros(2 * N, dtype=torch.int32)[::2]]
    for x in good:
        if not isinstance(x, int):
            assert x.data_ptr() % 16 == 0
        for name, call in _calls(m, x).items():
            assert call() in (eb.ECHO_ERR_NULL, eb.ECHO_ERR_HIP), name
    for x in bad:
        for name, call in _calls(m, x).items():
            with pytest.raises(ValueError):
                call()
                pytest.fail(f"{name} took {x.dtype}, {tuple(x.shape)}")
    for name, call in _calls(m, None).items():
        assert call() in (eb.ECHO_ERR_NULL, eb.ECHO_ERR_HIP), name
