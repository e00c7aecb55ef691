"""Without a GPU: how the products of the operators that keep nothing between the passes are cut, as far as their workspaces' sizes show it."""
from paper_2502_11034_amd import binding as B


def test_gradients_of_very_many_gated_columns_are_not_taken_in_parts():
    """Parts of rows that far apart have no tile: d_g and d_u are 4 bytes a value, not 6."""
    rows, dim = 128, 128
    for hidden in (2 ** 23, 2 ** 23 + 5, 2 ** 25):
        values = rows * hidden
        assert 2 * 4 * values <= B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, B.ADAGC_F32) < 2 * 4 * values + 2 ** 28
    hidden = 2 ** 23 - 64
    assert B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, B.ADAGC_F32) >= 2 * 6 * rows * hidden


def test_projections_have_no_more_partial_sums_than_their_documentation_says():
    """2^25 bytes at most, beside a row's parts (8 bytes for 32 tokens or more of it, and its target); few large tiles, which are not shared out, have none."""
    for rows in (1, 17, 56, 128, 300, 1024, 2048, 2049, 4096):
        for dim in (64, 768, 2048, 4096, 16384):
            for wide in (64, 1000, 2048, 4096, 14336):
                assert B.adagc_gated_linear_workspace_bytes(rows, dim, wide, B.ADAGC_BF16) <= 2 ** 25, (rows, dim, wide)
                parts = 8 * rows * (wide // 32 + 2) + 4 * rows + 32
                assert B.adagc_linear_logprobs_workspace_bytes(rows, wide, dim, B.ADAGC_BF16) <= 2 ** 25 + parts, (rows, dim, wide)
    assert B.adagc_gated_linear_workspace_bytes(1024, 4096, 4096, B.ADAGC_BF16) == 0                       # 128 tiles of 256 x 256
    assert B.adagc_linear_logprobs_workspace_bytes(2048, 4096, 4096, B.ADAGC_BF16) < 2 ** 20


def test_operands_that_one_launch_cannot_lay_out_are_too_large():
    """bf16 rows of no whole vectors, laid out anew in one launch of 2^32 lanes, 8 numbers each, at most: x of 5824 rows and both weights of 2912, each within its own
    limit, are more."""
    for f in (B.lib().adagc_gated_linear_workspace_bytes, B.lib().adagc_gated_linear_backward_workspace_bytes):
        assert f(5824, 46000 * 64 - 3, 2912, B.ADAGC_BF16) == B.ADAGC_ERR_TOO_LARGE
        assert f(5824, 45500 * 64 - 3, 2912, B.ADAGC_BF16) > 0
        assert f(5824, 46000 * 64, 2912, B.ADAGC_BF16) >= 0              # as they are
