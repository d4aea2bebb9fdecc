"""The temperatures that the operators behind the classifier take, without a GPU: 2^-126 to 2^126, as the header says."""
import pytest

from paper_1805_12549_amd import binding as B

CALLS = {
    "logprobs": lambda t: B.cg_logprobs(0, B.CG_F32, 0, 10, 10, t, 0, 0, 0, 0, 0, 0, 0, 0, 0),
    "forward": lambda t: B.cg_distill_forward(0, B.CG_BF16, 0, 10, 10, t, 0, 0, 0, 0, 0.0, 0.0, 0, 0, 0, 0, 0, 0, 0),
    "backward": lambda t: B.cg_distill_backward(0, B.CG_F32, 0, 10, 10, t, 0, 0, 0, 0, 0.0, 0.0, 0, 0, 0, 0),
}


@pytest.mark.parametrize("call", CALLS)
def test_temperatures(call):
    for taken in (2.0 ** -126, 2.0 ** -100, 1.0, 2.0 ** 126):
        CALLS[call](taken)                # (no rows: nothing is enqueued)
    for refused in (2.0 ** -127, 2.0 ** -130, 2.0 ** 127, 1.5 * 2.0 ** 126):
        with pytest.raises(B.CGError) as e:
            CALLS[call](refused)
        assert e.value.code == B.CG_EINVAL
