"""What the helpers that describe tensors to the calls say of a tensor that they cannot."""
import pytest
import torch

from paper_2411_12780_amd import binding as P

E = torch.zeros(4, dtype=torch.int8)


@pytest.mark.parametrize("call,what", [(lambda t: P.rows(t), "rows are 2-d tensors"), (lambda t: P.byte_rows(t, E), "rows of 8 bits are 2-d tensors"),
                                       (lambda t: P.queries_keys(t, None), "queries and keys are 2-d tensors"),
                                       (lambda t: P.queries_keys(None, t), "queries and keys are 2-d tensors")])
@pytest.mark.parametrize("shape", ["three axes", "turned"])
def test_the_message_names_what_was_given(call, what, shape):
    t = torch.zeros(4, 16, 2, dtype=torch.int8) if shape == "three axes" else torch.zeros(16, 4, dtype=torch.int8).t()
    with pytest.raises(P.PpllError) as e:
        call(t)
    assert e.value.status == 3 and what in str(e.value), str(e.value)
