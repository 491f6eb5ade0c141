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


def _ffn_args(device="cpu", T=6, K=2, D=64, E=4, F=128):
    e = lambda *s, d=torch.bfloat16: torch.empty(*s, dtype=d, device=device)  # noqa: E731
    n, i32, f32 = T * K, torch.int32, torch.float32
    fwd = dict(x_perm=e(n, D), expert_offsets=e(E + 1, d=i32), w1=e(E, 2 * F, D), w2=e(E, D, F),
               h_q=e(n, 2 * F, d=torch.int8), h_scale=e(2 * F // 32, n, d=f32), y_perm=e(n, D), ws=None)
    bwd = dict(dy=e(T, D), x=e(T, D), prob_perm=e(n, d=f32), row_of_slot=e(T, K, d=i32),
               **{k: fwd[k] for k in ("expert_offsets", "h_q", "h_scale", "w1", "w2")}, dx_perm=e(n, D),
               dw1=e(E, 2 * F, D), dw2=e(E, D, F), dprob_perm=e(n, d=f32), ws=None)
    return dict(S=T, GBS=1, K=K, D=D, E=E, F=F), fwd, bwd


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_ckpt_ffn_tensors(L, which, monkeypatch):
    """Every tensor of another type or size, and the scales as [rows, blocks], are refused by name."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    shape, fwd, bwd = _ffn_args()
    s = L.MoeShape.of(**shape)
    fn, args = (L.moe_expert_ffn_ckpt, fwd) if which == "forward" else (L.moe_expert_ffn_bwd_ckpt, bwd)
    for k, t in args.items():
        if t is None:
            continue
        bad = [t[:-1]] if t.dim() == 1 or k in ("dy", "x") else [t[:, :-1]]
        if k not in ("dw1", "dw2"):  # fp32 or bf16
            bad += [t.double(), t.long()]
        if t.dim() > 1 and k != "row_of_slot":
            bad.append(t.transpose(-1, -2).contiguous())
        for b in bad:
            with pytest.raises(ValueError, match=f"{k} is"):
                fn(s, **{**args, k: b}, stream=0)


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_ckpt_ffn_devices(L, which):
    shape, fwd, bwd = _ffn_args()
    s = L.MoeShape.of(**shape)
    fn, args = (L.moe_expert_ffn_ckpt, fwd) if which == "forward" else (L.moe_expert_ffn_bwd_ckpt, bwd)
    args["ws"] = torch.empty(256, dtype=torch.uint8)
    first = ("dw1", "dw2")  # they are asked for their type, and come before these two
    for k, t in args.items():  # the others as addresses
        rest = {n: v if n in first else 0x10000 for n, v in args.items()}
        name = "dw1" if which == "backward" and k in ("dprob_perm", "ws", "dw2") else k
        with pytest.raises(ValueError, match=f"{name} is on cpu"):
            fn(s, **{**rest, k: t}, stream=0)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_ckpt_rows_off_the_gpu(L, dt):
    x, q, s = torch.zeros(4, 64, dtype=dt), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(2, 4)
    with pytest.raises(ValueError, match="is on cpu"):
        L.moe_ckpt_pack(x, q, s, stream=0)
    with pytest.raises(ValueError, match="is on cpu"):
        L.moe_ckpt_unpack(q, s, x, stream=0)


def test_few_tokens_odd_rows_of_w1(L):
    """w1 has gate and up rows in pairs; with 2F + 1 rows an expert's weights would be read a row off."""
    from paper_2608_28511_gb300.layer import FewTokens
    bf = torch.bfloat16
    with pytest.raises(ValueError, match="w1"):
        FewTokens(torch.zeros(8, 128, dtype=bf), torch.zeros(8, 129, 128, dtype=bf), torch.zeros(8, 128, 64, dtype=bf), 2)
