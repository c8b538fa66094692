"""The batch calls' streams, as far as that can be seen without a GPU."""
import types

import pytest
import torch

from paper_2505_16162_amd import binding


def test_a_stream_of_another_gpu_is_refused_before_anything_is_launched():
    other = types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=1)
    called = []
    with pytest.raises(ValueError, match="stream must be one of cuda:0"):
        binding._call(torch.device("cuda:0"), other, (), lambda *a: called.append(a))
    with pytest.raises(ValueError, match="stream must be one of"):
        binding._output(torch.empty(2), other)
    assert not called
