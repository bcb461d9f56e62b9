"""The binding of the layer steps, checkpoints and label heads at its own limits (no GPU): counts
beyond 32 bits."""

import pytest
import torch

from paper_1812_04352_amd import lp as L


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 8, 2 ** 63])
def test_counts_beyond_32_bits_are_refused(n):
    """They do not fit the descriptors' fields, which would keep their low 32 bits: a step of 2^32 + 8
    rows must not run as one of 8, nor one of 2^32 rows as an empty one."""
    for make in (lambda: L.step("bf16", "tanh", n, 16, 16), lambda: L.step("bf16", "tanh", 8, n, 16),
                 lambda: L.step("bf16", "tanh", 8, 16, n)):
        with pytest.raises(L.LpError):
            L.lp_step_workspace_bytes(make())
    for make in (lambda: L.label_head("bf16", n, 16, 100), lambda: L.label_head("bf16", 8, n, 100),
                 lambda: L.label_head("bf16", 8, 16, n)):
        with pytest.raises(L.LpError):
            L.lp_loss_labels_workspace_bytes(make(), True)
    assert L.step("bf16", "tanh", -n, 16, 16).B < 0


class Rows:
    """A tensor of `rows` rows of one feature, as far as the binding looks."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, rows, dtype):
        self.rows, self.dtype = rows, dtype
        self.shape = (rows, 1)

    def dim(self):
        return 2

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def numel(self):
        return self.rows

    def data_ptr(self):
        return 1 << 20 if self.dtype == torch.bfloat16 else 1 << 21 if self.dtype == torch.int8 else 1 << 22


def test_checkpoints_of_more_rows_than_32_bits_count(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(L, "_stream_of", lambda dev: None)
    for n in (2 ** 31, 2 ** 32):
        x, x8, xe = (Rows(n, t) for t in (torch.bfloat16, torch.int8, torch.uint8))
        for call in (lambda: L.lp_checkpoint_store(x, x8, xe), lambda: L.lp_checkpoint_load(x8, xe, x)):
            with pytest.raises(L.LpError) as e:
                call()
            assert e.value.status == L.LP_EUNSUPPORTED


def test_first_calls_of_two_threads(monkeypatch):
    """While one thread's first call fills the table of dtypes, another's finds it empty or whole."""
    seen = []

    class Watched(dict):
        def __setitem__(self, k, v):
            super().__setitem__(k, v)
            if not seen:
                seen.append(None)
                seen.append(L._wide_dtype(L.LP_BF16))  # what a call between two entries gets

    monkeypatch.setattr(L, "_torch_dtypes", Watched())
    assert L._wide_dtype(L.LP_BF16) == torch.bfloat16
    assert seen in ([], [None, torch.bfloat16])
