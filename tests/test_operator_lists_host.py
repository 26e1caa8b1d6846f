"""Lists of tensors that change while a call reads them, in a process of its own: a tensor's methods may be any code."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import gc
import torch
import paper_2107_14575_amd as dq


class Tensor:
    '''What a call asks of a tensor; asked for its type, it empties the list that it is in.'''
    def __init__(self, of):
        self.of = of
    @property
    def dtype(self):
        self.of.clear()
        gc.collect()
        junk = [[k] * 8 for k in range(4096)]  # where the list's items were
        return torch.float32
    def is_contiguous(self):
        return True
    def get_device(self):
        return 0
    def numel(self):
        return 4
    def data_ptr(self):
        return 4096


grads = []
grads.extend(Tensor(grads) for _ in range(50))
call = {"norm": lambda: dq.grad_norm(grads, None, None), "clip": lambda: dq.clip_grads(grads, 1.0, None, None), "out": lambda: dq.clip_grads([], 1.0, None, None, out=grads)}
try:
    call[WHICH]()
except (AttributeError, ValueError) as e:  # of the norm, which is no tensor, or of the sizes: nothing is launched
    print("refused", type(e).__name__)
"""


@pytest.mark.parametrize("which", ["norm", "clip", "out"])
def test_a_list_that_changes(which):
    r = subprocess.run([sys.executable, "-c", PROGRAM.replace("WHICH", repr(which))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("refused"), (r.returncode, r.stdout, r.stderr[-2000:])
