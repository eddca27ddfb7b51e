"""What a step refuses to say of its tokens, before anything is launched: numbers of alternatives that the calls below it refuse."""
import pytest

torch = pytest.importorskip("torch")

import paper_2601_12212_amd as dt  # noqa: E402
from paper_2601_12212_amd.step import Step  # noqa: E402


def test_numbers_of_alternatives_that_are_none():
    st = Step([(8, 2, 3), (6, 3, 2)], [4, 0], 4, 2, 64, 100, device="cpu")
    for call, k in ((st.draft_loss, 0), (st.draft_loss, -1), (st.token_logprobs, -1)):
        with pytest.raises(dt.DtError) as e:
            call(k)
        assert e.value.status == -1
    assert not st._buffers
