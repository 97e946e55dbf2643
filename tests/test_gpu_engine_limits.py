"""Sizes at the ends of what the arguments' types hold: refused before anything is launched."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("rows", [2 ** 30 + 1, 2 ** 31 - 256, 2 ** 31 - 1])
def test_products_of_more_rows_than_tiles_can_count(ctx, rows):
    L, at = binding.lib(), torch.zeros(4096, dtype=torch.int8, device=DEV).data_ptr()
    assert L.dropmatch_matmul_i8(ctx._h, at, 16, at, rows, at, 16, at, 1, 16, at, binding.F32, 1, None) == binding.EUNSUPPORTED
    assert L.dropmatch_linear_i8(ctx._h, at, binding.F32, 16, rows, at, 16, at, 1, 16, at, 16, at, at, binding.F32, 1, None) == binding.EUNSUPPORTED


@pytest.mark.parametrize("B,T,bonus", [(1, 2 ** 31 - 1, 1), (1, 2 ** 31 - 1, 0), (1, 2 ** 27, 1), (2 ** 27 + 1, 0, 1), (2 ** 20, 128, 1)])
def test_more_positions_than_one_launch_takes(ctx, B, T, bonus):
    L, at = binding.lib(), torch.zeros(4096, dtype=torch.int8, device=DEV).data_ptr()
    assert L.dropmatch_verify_lossless(ctx._h, at, binding.F32, 8, None, binding.F32, 8, at, None, B, T, bonus, 8, 1.0, 1.0, at, at, at, at, at,
                                       None) == binding.EUNSUPPORTED
