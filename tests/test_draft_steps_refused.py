"""Steps of decoder blocks whose tensors have no rows to count: refused as other shapes are, with everything as it was (CPU only)."""
import pytest
import torch

from test_decoder_sequences import X, block, refused, taken


@pytest.mark.parametrize("tokens", [torch.zeros((), dtype=torch.bfloat16), torch.zeros(16, dtype=torch.bfloat16), torch.zeros(1, 2, 16, dtype=torch.bfloat16)])
def test_tokens_of_another_shape_are_refused_as_such(tokens):
    b = block()
    b.device = "cpu"
    taken(b, [[("a", X(60))], [("b", X(3))]])
    refused(b, [[("a", X(1))], [("b", tokens)]], ValueError)
    refused(b, [[("new", tokens)], []], ValueError)
    with pytest.raises(ValueError):
        b.step([[("a", tokens)], []], [{"a": [-1]}, None])
    assert b.sequences[0]["a"][1] == 60 and not any(b.drafts)


@pytest.mark.parametrize("logits", [torch.zeros(()), torch.zeros(2), torch.zeros(2, 3, 1)])
def test_logits_of_another_shape_are_refused_as_such(logits):
    b = block()
    b.device = "cpu"
    b._commit(b._admit([[("a", X(2))], []]), b._trees([[("a", X(2))], []], [{"a": [-1, 0]}, None]))
    with pytest.raises(ValueError, match="service 0"):
        b.accept([{"logits": logits, "tokens": torch.zeros(2, dtype=torch.int32), "uniforms": torch.zeros(2)}, None], [[1.0], []])
    assert b.drafts[0] == {"a": (0, [-1, 0])}
