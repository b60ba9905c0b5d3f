"""What the operators of a residual block and the orthogonalised rule lay out and refuse before anything is launched; no GPU needed."""
import pytest

from paper_1908_11848_amd import binding as B, residual_mlp as R


def test_workspaces_are_zero_for_what_is_refused_and_grow_with_the_sizes():
    L = B.lib()
    assert L.dsspk_layernorm_bwd_scratch_floats(5, 0) == L.dsspk_layernorm_bwd_scratch_floats(-1, 8) == L.dsspk_layernorm_bwd_scratch_floats(5, 16385) == 0
    assert L.dsspk_layernorm_bwd_scratch_floats(1, 100) == 0 and L.dsspk_layernorm_bwd_scratch_floats(10 ** 6, 100) == 2 * 100 * 1024
    for f in (L.dsspk_linear_fwd_workspace_bytes, L.dsspk_linear_bwd_workspace_bytes):
        for bad in ((2, 4, 4, 4), (0, -1, 4, 4), (0, 4, 0, 4), (0, 4, 4, 0), (0, 2 ** 31, 4, 4), (0, 4, 2 ** 20 + 1, 4)):
            assert f(*bad) == 0, bad
        # fp32 operands are six bytes a number, padded to 32 in a row
        assert f(0, 100, 33, 33) >= 6 * (100 * 64 + 33 * 64) and f(1, 0, 8, 8) > 0
        assert f(0, 2000, 64, 64) > f(0, 1000, 64, 64)


@pytest.mark.parametrize("matrices,fine", [([], True), ([(0, 8, 9)], True), ([(0, 8, 9), (72, 3, 3)], True), ([(0, 8, 9), (71, 3, 3)], False), ([(5, 0, 3)], False),
                                           ([(5, 3, -3)], False), ([(-1, 3, 3)], False), ([(0, 2 ** 20 + 1, 2)], False), ([(0, 16385, 16385)], False)])
def test_matrices_are_ascending_disjoint_and_not_empty(matrices, fine):
    assert (B.dssp_orthogonal_workspace_bytes(matrices) > 0) == fine


def test_a_networks_matrices_cover_its_weights():
    seg = R.segments(24, 40, 3, 10)
    mats = B.weight_matrices([s[1:] for s in seg])
    assert [(r, c) for _, r, c in mats] == [(48, 24)] + [(24, 40), (40, 24)] * 3 + [(24, 10)]
    assert B.dssp_orthogonal_workspace_bytes(mats) > 0
    segs = B.dssp_model_segments(B.model_id("alexnet_ds"), 10)
    assert [(r, c) for _, r, c in B.weight_matrices(segs)] == [(75, 64), (1600, 64), (3136, 384), (384, 192), (192, 10)]


def test_host_only_context_has_no_rule():
    ctx = B.dssp_create(None, 0, 2, 1, 1, 0.1)
    with pytest.raises(B.DsspError) as e:
        B.dssp_set_orthogonal_update(ctx, [(0, 2, 2)], 0.1, 16, 256, 1 << 20)
    assert e.value.code == B.DSSP_ESTATE
    B.dssp_destroy(ctx)


@pytest.mark.parametrize("matrices", [[(2 ** 63 - 1, 3, 3)], [(2 ** 63 - 9, 3, 3)], [(0, 2, 2), (2 ** 63 - 8, 3, 3)], [(2 ** 63 - 9, 3, 3), (5, 3, 3)]])
def test_matrices_whose_end_passes_64_bits_are_refused(matrices):
    """offset + rows * cols wraps round and would look as if it were within the vector"""
    assert B.dssp_orthogonal_workspace_bytes(matrices) == 0
    table = B.matrix_table(matrices)
    assert B.lib().dsspk_orthogonal_workspace_bytes(table, len(matrices)) == 0
    # refused by its arguments, in front of any launch (the addresses are never used)
    assert B.lib().dsspk_orthogonal_apply(None, 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 100, table, len(matrices), 0.1, 0.1, 0.9, 1, 5, 1e-7, 6 << 20, 1 << 60) == -1


@pytest.mark.parametrize("type", [0, 1])
def test_results_of_more_tiles_than_a_launch_has_are_refused(type):
    """by their sizes, in front of any launch (the addresses are never used)"""
    L, at, big = B.lib(), 1 << 20, 1 << 62
    n = 1 << 20
    assert L.dsspk_linear_bwd(None, type, at, n, at, 2 * at, n, None, 0, None, 0, 0, 3 * at, 4 * at, 4, n, n, 5 * at, big) == -1        # dw
    assert L.dsspk_linear_bwd(None, type, None, 0, at, 2 * at, 8, 3 * at, n, None, 0, 0, None, 4 * at, 1 << 30, 8, n, 5 * at, big) == -1       # dx
    assert L.dsspk_linear_fwd(None, type, at, 8, 2 * at, None, 0, None, 0, 3 * at, n, None, 0, 1 << 30, n, 8, 5 * at, big) == -1


def test_few_rows_need_no_workspace_of_the_weights_size():
    """A row through 8192 x 8192 in fp32 takes the weights as they are, not 400 MB of terms; more rows than that way serves take the terms."""
    f = B.lib().dsspk_linear_fwd_workspace_bytes
    assert all(0 < f(0, m, 8192, 8192) <= 1024 for m in (0, 1, 16)) and f(0, 17, 8192, 8192) >= 6 * 8192 * 8192
    assert all(0 < f(1, m, 4096, 1024) <= 1024 for m in (0, 1, 8)) and f(1, 9, 4096, 1024) >= 2 * 4096 * 1024


def test_the_products_of_the_tests_take_every_tile_there_is():
    import test_gpu_operator_tiles as tiles
    assert all(B.linear_form(tiles.linear.TYPE[f[0]], *f[1:4]) == f[4] for f in tiles.FORMS)
    one, many = ({(str(f[0]),) + f[4][:2] for f in tiles.FORMS if (f[4][2] > 1) == split} for split in (False, True))
    large = {("torch.bfloat16", 256, 256), ("torch.float32", 128, 128), ("torch.float32", 128, 64)}
    assert large <= one and large <= many
    # the small tiles are what most other sizes take
    assert B.linear_form(1, 300, 300, 72) == (128, 128, 1) and B.linear_form(0, 300, 300, 72)[:2] == (64, 64)
    with pytest.raises(ValueError):
        B.linear_form(0, 0, 3, 3)
