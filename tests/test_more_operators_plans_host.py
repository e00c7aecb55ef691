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
