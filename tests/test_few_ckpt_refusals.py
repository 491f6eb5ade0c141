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
    """Two devices of one kind are two devices (meta tensors keep the index they are given)."""
    from paper_2608_28511_gb300.layer import LayerScratch, MoeLayer
    base = dict(S=64, GBS=1, K=2, D=128, E=8, F=64)
    sc = LayerScratch(L.MoeShape.of(**base), "meta:0")
    same = MoeLayer(**base, device="meta:0", checkpoint="int8", scratch=sc)
    assert same.x_perm is sc.x_perm
    for device in ("meta:1", "cpu"):
        with pytest.raises(ValueError, match="scratch"):
            MoeLayer(**base, device=device, checkpoint="int8", scratch=sc)
