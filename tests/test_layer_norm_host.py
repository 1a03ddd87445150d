"""What can be seen of the layer norm without a GPU: the forms of its kernels that the library holds, sizes of workspaces."""
import re


def test_teams_that_sum_the_weights_gradients_have_eight_waves_at_most():
    """Their workgroups are eight waves; a form of a team of sixteen could not be launched."""
    from paper_2601_16991_amd import build
    with open(build.LIB, "rb") as f:
        forms = set(re.findall(rb"layer_norm_backward_kernelILb([01])ELi(\d+)ELi(\d+)ELb([01])ELb1EE", f.read()))
    assert {(int(team), int(units)) for _, team, units, _ in forms} == {(1, 1), (1, 2), (2, 2), (4, 2), (8, 2), (8, 4), (8, 8)}
    assert len(forms) == 28   # both types, rows of whole vectors and others


def test_workspace_of_few_rows_is_small():
    """Up to 512 rows one launch forms dx, dw and db and keeps no sums: the calls ask for two rows of them at most, not for those of 256 workgroups."""
    import paper_2601_16991_amd as salr
    for K in (1, 77, 4096, 32768):
        for T in (1, 8, 255, 512):
            assert 0 < salr.salr_layer_norm_backward_workspace_bytes(T, K, True) <= 8 * K, (T, K)
        assert salr.salr_layer_norm_backward_workspace_bytes(4096, K, True) == 256 * 8 * K
        assert salr.salr_layer_norm_backward_workspace_bytes(512, K, False) == 0
