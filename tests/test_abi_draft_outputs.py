"""The words and numbers that echo_draft_verify writes are torch.int32 tensors as large as what it writes; others are refused by both forms of the call,
without a GPU."""
import pytest

from test_abi_index_types import FORMS

A = 0x10000  # a fake, aligned, never dereferenced device address


def _verify(m, desc, **given):
    given = {**dict(drafted=A, n_drafted=A, draft=None, target=A, u=A, r=A, tokens=A, taken=A, workspace=A, workspace_bytes=1 << 60), **given}
    return m.echo_draft_verify(desc, **given)


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("name,count", [("tokens", 15), ("taken", 3)])
def test_output_tensors(form, name, count):
    import torch
    m = FORMS[form]()
    d = m.make_draft_desc(3, 4, 9)
    for x in (torch.zeros(count, dtype=torch.int32), torch.zeros(2, count, dtype=torch.int32), A):
        assert _verify(m, d, **{name: x}) == m.ECHO_ERR_NULL                  # taken, and then stopped at `draft`
    assert _verify(m, d, draft=A, **{name: None}) == m.ECHO_ERR_NULL
    for x in (torch.zeros(count, dtype=torch.int64), torch.zeros(count), torch.zeros(count - 1, dtype=torch.int32),
              torch.zeros(2 * count, dtype=torch.int32)[::2], torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError):
            _verify(m, d, **{name: x})
            pytest.fail(f"{name} took {x.dtype}, {tuple(x.shape)}")


@pytest.mark.parametrize("form", sorted(FORMS))
def test_descriptors_that_are_refused_ask_for_nothing(form):
    import torch
    m = FORMS[form]()
    for field in ("B", "K", "V"):
        for value in (0, -1, -2 ** 31, 2 ** 31 - 1):
            d = m.make_draft_desc(3, 4, 9)
            setattr(d, field, value)
            if field != "V" and value == 2 ** 31 - 1:                       # more words than the tensors have: refused by their size
                with pytest.raises(ValueError):
                    _verify(m, d, tokens=torch.zeros(15, dtype=torch.int32))
                continue
            assert _verify(m, d, tokens=torch.zeros(15, dtype=torch.int32), taken=torch.zeros(3, dtype=torch.int32)) == m.ECHO_ERR_SHAPE
