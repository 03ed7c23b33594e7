"""Host-side checks of the token-sequence operators' options: no GPU, no kernel is launched."""
import pytest

import test_abi_host
from paper_2412_06355_gb300 import binding


def test_logit_grad_is_checked():
    cfg = binding.make_xent_config(10, 20, 8, "bf16", logit_grad="bf16")
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 0
    cfg.logit_grad = 2
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    cfg = binding.make_xent_config(10, 20, 8, "f32", logit_grad="bf16")
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    with pytest.raises(ValueError, match="logit_grad"):
        binding.make_xent_config(10, 20, 8, "bf16", logit_grad="f16")
