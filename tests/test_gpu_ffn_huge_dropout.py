"""Dropout of more elements than one dimension of a grid has lanes for: 2^36 of 16 bits are 2^32 lanes of sixteen."""
import numpy as np
import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import ffn_ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def halves(first, count, seed, offset):
    """The upper 16 bits of the numbers of elements first .. first + count - 1, both multiples of eight."""
    index = np.arange(first // 8, (first + count) // 8, dtype=np.uint64)
    words = ffn_ref.philox((index & np.uint64(0xFFFFFFFF), index >> np.uint64(32), np.full_like(index, offset),
                            np.zeros_like(index)), (seed, 0))
    return np.stack([(words[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)], 1).reshape(-1)


def test_dropout_of_128_gigabytes_in_place():
    n = (1 << 36) + 4104
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 2 * n + (4 << 30):
        pytest.skip("less than 132 GB of GPU memory are free")
    say("dropout of %d bf16 elements" % n)
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    ffn.zvc_dropout(x, x, 0.5, 5, 6)
    torch.cuda.synchronize()
    count = 1 << 16
    for first in (0, (1 << 32) - count, 1 << 32, 1 << 35, (1 << 36) - count, 1 << 36, n - 4096):
        part = x[first:min(first + count, n)].cpu()
        want = torch.from_numpy(halves(first, part.numel(), 5, 6) >= 0x8000)
        assert torch.equal(part, want.to(part.dtype) * 2), first
    del x
    torch.cuda.empty_cache()
