"""A gradient's workspace serves every smaller batch: its size does not fall as positions, values or rows grow, and what was measured for the
largest batch is enough for the last one of an epoch."""
import random

import pytest
import torch

from paper_1804_08066_amd import mqgrad as mq
from test_gpu_embedding import BF16, DEV, check_grad, matrix, some_tokens


def sizes_grow(points):
    L = mq.lib()
    before = None
    for at in points:
        need = L.mqg_embedding_grad_workspace_bytes(*at)
        assert before is None or need >= before[1], (before, at, need)
        before = (at, need)


@pytest.mark.parametrize("rows", [1, 15, 16, 1023, 1024, 50257, (1 << 20) + 1])
@pytest.mark.parametrize("dim", [1, 8, 9, 64, 65, 128, 1000, 2048, 2049, 4096, 20000])
def test_sizes_grow_with_the_positions(dim, rows):
    sizes_grow((n, dim, rows) for n in range(1, 5000))
    for at in (8192, 16384, 16385, 32768, 65536, 131072, 262144, 524288, 1 << 20):
        sizes_grow((n, dim, rows) for n in range(at - 130, at + 130))
    sizes_grow((n, dim, rows) for n in range(5000, 600_000, 127))


@pytest.mark.parametrize("count", [1, 256, 257, 4096, 4097, 8192, 16384, 70_000, 1 << 20])
def test_sizes_grow_with_the_values_and_the_rows(count):
    for rows in (1, 16, 50257):
        sizes_grow((count, dim, rows) for dim in range(1, 5000))
    for dim in (1, 16, 1000, 4096):
        sizes_grow((count, dim, rows) for rows in range(1, 5000))
        sizes_grow((count, dim, 1 << k) for k in range(31))


def test_a_size_holds_for_every_smaller_batch():
    rnd = random.Random(5)
    limits = (1 << 22, 1 << 20, 1 << 30)
    L = mq.lib()
    for _ in range(100_000):
        large = [max(1, int(2 ** rnd.uniform(0, limit.bit_length() - 1))) for limit in limits]
        small = [max(1, int(x * 2 ** -rnd.uniform(0, 3))) for x in large]
        assert L.mqg_embedding_grad_workspace_bytes(*small) <= L.mqg_embedding_grad_workspace_bytes(*large), (small, large)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,rows,largest,counts", [(4096, 500, 8192, [8191, 5000, 1]), (64, 700, 33_000, [32_767, 16_385, 16_384, 4097, 300]),
                                                      (16, 40, 131_072, [131_071, 65_535]), (16, 16, 4096, [4000, 300])])
def test_one_workspace_for_batches_of_all_lengths(dim, rows, largest, counts):
    need = mq.mqg_embedding_grad_workspace_bytes(largest, dim, rows)
    memory = torch.full((need + 65536,), 0xA5, dtype=torch.uint8, device=DEV)
    for count in [largest, *counts]:
        for few in (rows, max(1, rows - 1)):
            g = matrix(count, dim, count, BF16)
            ids = some_tokens("text", count, few, seed=count).to(DEV)
            out = torch.full((few, dim), 9.0, device=DEV)
            mq.mqg_embedding_grad(g, ids, few, out=out, workspace=memory[:need])
            check_grad(g, ids, out, few, 1.0)
            assert (memory[need:] == 0xA5).all()
