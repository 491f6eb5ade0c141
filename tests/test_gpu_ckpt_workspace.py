"""The checkpointed FFN's workspace at any 16-byte alignment, which is all that the interface asks for."""
import pytest
import torch

from tests.test_gpu_ckpt import _backward, _case, _device, _forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("off", [16, 32, 64, 112, 128, 240])
def test_workspace_alignment(off):
    """The same bits as from a 256-byte aligned workspace, and nothing written outside it."""
    from paper_2608_28511_gb300 import abi
    w, inp, offs, ros, tor, pp = _case("uneven")
    s, d = _device(w, inp, offs, ros, tor, pp)
    n = abi.moe_ckpt_workspace_size(s)
    assert d["ws"].data_ptr() % 256 == 0
    want = _forward(w, s, d)
    want += _backward(w, s, d, want[0], want[1])
    buf = torch.full((n + 1024,), 255, dtype=torch.uint8, device="cuda")
    assert buf.data_ptr() % 256 == 0
    d["ws"] = buf[off:off + n]
    got = _forward(w, s, d)
    got += _backward(w, s, d, got[0], got[1])
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert (buf[:off] == 255).all() and (buf[off + n:] == 255).all()
