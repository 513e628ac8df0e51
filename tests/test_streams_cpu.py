"""The stream that a call is given: no GPU is needed for what is refused."""
from types import SimpleNamespace

import pytest
import torch

from paper_1502_00512_amd import binding


def test_a_stream_of_another_device_is_refused():
    def call():
        raise AssertionError("called")

    with pytest.raises(binding.RnnlmError, match="stream: one of device 0"):
        binding._on("rnnlm_top_logits", SimpleNamespace(device=torch.device("cuda", 1)), 0, call)
