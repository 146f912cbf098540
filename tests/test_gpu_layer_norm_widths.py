"""Layer norm at the widths where the number of threads and packs that hold a row changes, one below, at and above it, with rows that
end inside a pack, and one beyond what is held at all."""
import pytest
import torch

from test_gpu_layer_norm import TYPES, run

pytestmark = pytest.mark.gpu

PACK = {"f32": 4, "bf16": 8, "f16": 8}
# packs: 64, 128, 256, 512 threads with one; 64 with up to 4 (forward); 256, 512, 1024 with up to 4
STEPS = [64, 128, 192, 256, 512, 768, 1024, 1536, 2048, 3071, 4096]


@pytest.mark.parametrize("dtype,w", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("packs", STEPS)
def test_around_a_step(packs, dtype, w):
    for cols in (packs * PACK[dtype] - 1, packs * PACK[dtype], packs * PACK[dtype] + 1):
        run(7, cols, TYPES[dtype], TYPES[w])


@pytest.mark.parametrize("rows", [1, 2, 3, 8, 511, 512, 513, 1025, 4100])
@pytest.mark.parametrize("cols", [500, 1000, 2000, 4000])
def test_rows_that_do_not_fill_the_groups(rows, cols):
    run(rows, cols, torch.bfloat16, torch.float32)
