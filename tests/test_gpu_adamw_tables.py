"""AdamW over numbers of tensors on both sides of what one launch holds: the same step as tensor by tensor, hash and all."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit
from tests.test_gpu_adamw import make, run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [1, 191, 192, 193, 447, 448, 449, 640, 641, 900])
@pytest.mark.parametrize("bits", [8, 32])
def test_every_number_of_tensors(count, bits):
    sizes = [(i * 53) % 700 for i in range(count)]
    run_and_check(make(sizes, torch.bfloat16, torch.float32, bits, False, count), bits, step=3, seed=11)
