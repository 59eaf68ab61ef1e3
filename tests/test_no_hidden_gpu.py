"""Where torch sees no GPU the library sees none either: tests that need no GPU call it with invented addresses."""
import os

import torch


def test_the_library_sees_no_gpu_that_torch_does_not_see():
    assert torch.cuda.is_available() or os.environ["HIP_VISIBLE_DEVICES"] == "-1"
