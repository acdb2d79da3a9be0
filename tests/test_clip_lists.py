"""Lists of gradients that dynb_clip_gradients would scale twice at one place are refused ahead of any launch (no GPU is needed)."""
import pytest
import torch

from paper_1707_02402_amd import binding


class Tensor:
    is_cuda, dtype = True, torch.float32

    def __init__(self, at, n=4):
        self.at, self.n = at, n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n


def test_results_at_one_place_are_refused():
    a, b, c = Tensor(4096), Tensor(8192), Tensor(16384)
    with pytest.raises(AssertionError):
        binding.GradTensors([a, b, a])                                 # tied parameters, listed by both names
    with pytest.raises(AssertionError):
        binding.GradTensors([a, b], [c, c])
    assert len(binding.GradTensors([a, a], [b, c]).array) == 2         # (read twice, written apart)
    empty = binding.GradTensors([a, Tensor(0, 0), b, Tensor(0, 0)])
    assert [t.grad for t in empty.array] == [4096, None, 8192, None] and [t.count for t in empty.array] == [4, 0, 4, 0]
