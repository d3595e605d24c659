"""The training operators' tests get the same inputs in every process (no GPU)."""
import os
import subprocess
import sys

import torch

from tests import conftest, ffn_inputs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
from tests import conftest, test_gpu_ffn
test_gpu_ffn.DEV = "cpu"
with conftest.repeatable_inputs(test_gpu_ffn):
    print([test_gpu_ffn.generator(33, "torch.float16", *more).initial_seed() for more in ((), ("directions",))])
"""


def drawn(salt):
    env = dict(os.environ, PYTHONHASHSEED=salt)
    done = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    return done.stdout


def test_seeds_do_not_depend_on_the_process():
    assert drawn("1") == drawn("2")


def test_seeds_differ_by_every_part_of_the_key():
    keys = [(1, 2), (2, 1), (12,), ("1", 2), (1, "torch.float16"), (1, "torch.bfloat16")]
    assert len({ffn_inputs.seed_of(*key) for key in keys}) == len(keys)


def test_only_what_seeds_by_hash_is_replaced():
    class Module:
        generator = staticmethod(lambda *key: None)
    before = Module.generator
    with conftest.repeatable_inputs(Module):
        assert Module.generator is before
    assert torch.equal(torch.randn(3, generator=ffn_inputs.generator("a", device="cpu")),
                       torch.randn(3, generator=ffn_inputs.generator("a", device="cpu")))
