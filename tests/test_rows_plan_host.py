"""What the row operators plan, without a GPU: sizes of workspaces."""
import itertools

import pytest

from paper_2309_15812_amd import _lib, ops

F32, BF16 = 0, 1
NONE, GELU = 0, 2


def ln_bytes(M, C, dt):
    return _lib.lib().o1d_ln_bwd_workspace_bytes(M, C, dt)


def wgrad_bytes(M, I, O, dt, act=NONE, held=0):
    return _lib.lib().o1d_linear_bwd_weight_workspace_bytes(M, I, O, act, held, dt)


# Small calls whose partial results take 256 bytes or fewer: layer norm's backward in several workgroups, a
# weight gradient in several pieces.
SMALL_LN = [(513, 1), (513, 6), (4096, 1), (700, 3)]
SMALL_WGRAD = [(256, 7, 4, F32), (600, 1, 8, BF16)]


@pytest.mark.parametrize("M,C", SMALL_LN)
@pytest.mark.parametrize("dt", [F32, BF16])
def test_small_layer_norm_gradients_have_a_workspace_of_their_own(M, C, dt):
    # (one workgroup, which writes no partial results, has at most 4 x 64 / 4 x 8 = 512 rows of so few features)
    assert ln_bytes(M, C, dt) > ops._NO_SPACE


@pytest.mark.parametrize("M,I,O,dt", SMALL_WGRAD)
def test_small_weight_gradients_have_a_workspace_of_their_own(M, I, O, dt):
    assert wgrad_bytes(M, I, O, dt) > ops._NO_SPACE


def test_workspaces_are_nothing_or_larger_than_what_calls_share():
    sizes = [1, 2, 3, 5, 7, 8, 13, 31, 64, 97, 200, 256, 300, 513, 600, 1000, 2049, 4096, 9001]
    for M, C, dt in itertools.product(sizes, [1, 2, 3, 4, 5, 6, 8, 11, 24, 96, 700], [F32, BF16]):
        assert ln_bytes(M, C, dt) == ops._NO_SPACE or ln_bytes(M, C, dt) >= 2 * ops._NO_SPACE, (M, C, dt)
    for M, I, O, dt in itertools.product(sizes, [1, 2, 4, 7, 8, 24], [1, 3, 4, 8, 17], [F32, BF16]):
        for act, held in ((NONE, 0), (NONE, 1), (GELU, 0), (GELU, 1)):
            b = wgrad_bytes(M, I, O, dt, act, held)
            assert b == ops._NO_SPACE or b >= 2 * ops._NO_SPACE, (M, I, O, dt, act, held)


def test_the_tests_reach_every_kernel_that_is_planned():
    """A kernel that drawn calls take and no size of the GPU tests does: add a size for it (rows_cases.py)."""
    import rows_cases

    missing = {n: c for n, c in rows_cases.planned(40000).items() if n not in rows_cases.reached()}
    assert not missing, missing


def test_names_of_planned_kernels():
    def name(*args, **kw):
        return _lib.rows_kernel_name(*args, **kw)

    assert name("ln_fwd", 49, 768) == "ln_fwd/f32/64x3" and name("ln_bwd", 33333, 211, held=True, dtype=BF16).endswith("/held+col_sum")
    assert name("ln_fwd", 3, 9001) == "ln_fwd/f32/wide" and name("linear_fwd", 16, 768, 1000, dtype=BF16) == "few/fwd/bf16/16"
    assert name("linear_fwd", 20000, 768, 768, dtype=BF16).startswith("mmf/fwd/bf16/")
    assert name("linear_fwd", 20000, 768, 768, dtype=BF16, aligned=False).startswith("mm/fwd/bf16/")
    assert name("linear_bwd_weight", 50176, 768, 192, act="gelu", held=True, dtype=BF16).startswith("mm/wgrad/bf16/192x64/made+mm_sum")
    assert name("linear_bwd_weight", 8192, 2048, 2048, act="gelu", held=True, dtype=BF16).startswith("act+mmf/wgrad/")
    assert name("linear_fwd", 0, 8, 8) == name("linear_fwd", 8, 0, 8) == name("ln_fwd", 8, -1) == ""
    assert _lib.lib().o1d_rows_kernel_name(5, 8, 8, 8, 0, 0, F32, 1) == _lib.lib().o1d_rows_kernel_name(0, 8, 8, 8, 9, 0, F32, 1) == b""
