"""What the few-token layer and the checkpoint bindings refuse before any launch (no GPU needed)."""
import os
import shutil

import pytest
import torch

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                reason="nvcc is needed to build the library")


@pytest.fixture(scope="module")
def L():
    from paper_2608_28511_gb300 import _build, abi
    _build.build()
    return abi


def test_scratch_of_another_device(L):
    """Two GPUs are two devices (tensors without memory, which keep the device they are made for)."""
    from torch._subclasses.fake_tensor import FakeTensorMode

    from paper_2608_28511_gb300.layer import LayerScratch, MoeLayer
    base = dict(S=64, GBS=1, K=2, D=128, E=8, F=64)
    with FakeTensorMode(allow_non_fake_inputs=True):
        sc = LayerScratch(L.MoeShape.of(**base), "cuda:0")
        assert MoeLayer(**base, device="cuda:0", checkpoint="int8", scratch=sc).x_perm is sc.x_perm
        for device in ("cuda:1", "cpu"):
            with pytest.raises(ValueError, match="scratch"):
                MoeLayer(**base, device=device, checkpoint="int8", scratch=sc)
