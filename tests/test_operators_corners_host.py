"""Corners of the operators around the step that need no GPU."""
import pytest

from paper_2502_11034_amd import binding as B


def test_workspace_of_a_weight_gradient_that_is_refused():
    """The size of a workspace is refused where the call is: more tiles than a launch takes."""
    for n_out, n_in in ((2 ** 31 - 1024, 2 ** 31 - 1024), (2 ** 24, 2 ** 24)):
        with pytest.raises(B.AdagcError):
            B.adagc_act8_wgrad_workspace_bytes(1, n_out, n_in, B.ADAGC_BF16)
        assert B.lib().adagc_act8_wgrad(1 << 20, B.ADAGC_BF16, n_out, 1 << 20, 1, n_out, n_in, 1 << 21, B.ADAGC_F32, n_in, 0, None, 0,
                                        None) == B.ADAGC_ERR_TOO_LARGE
    for n_out, n_in in ((2 ** 31 - 1024, 1), (1, 2 ** 31 - 1024), (2 ** 29 + 1, 64)):
        for dtype in (B.ADAGC_F32, B.ADAGC_BF16):
            assert B.adagc_act8_wgrad_workspace_bytes(1, n_out, n_in, dtype) >= 0


def test_sizes_beyond_their_type_are_refused():
    """Not answered for what is left of them."""
    for call in (lambda: B.adagc_token_logprobs_workspace_bytes(1, 128256, 2 ** 32), lambda: B.adagc_token_logprobs_workspace_bytes(2 ** 64 + 1, 128256),
                 lambda: B.adagc_act8_bytes(2 ** 64 + 1, 32), lambda: B.adagc_act8_bytes(1, 2 ** 70),
                 lambda: B.adagc_act8_wgrad_workspace_bytes(1, 4, 5, 2 ** 32 + 1), lambda: B.adagc_act8_wgrad_workspace_bytes(-2 ** 64, 4, 5, 1)):
        with pytest.raises(B.AdagcError):
            call()
