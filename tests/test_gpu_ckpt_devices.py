"""The checkpoint bindings refuse a tensor that is not on the GPU, whichever it is, before any launch."""
import pytest
import torch

from tests.test_gpu_ckpt import _case, _device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def test_ffn_tensors_off_the_gpu():
    from paper_2608_28511_gb300 import abi
    w, inp, off, ros, tor, pp = _case("one_token")
    s, d = _device(w, inp, off, ros, tor, pp)
    e = lambda *n, t=torch.bfloat16: torch.zeros(*n, dtype=t, device="cuda")  # noqa: E731
    f32, n = torch.float32, w.TK
    fwd = dict(x_perm=d["x_perm"], expert_offsets=d["off"], w1=d["w1"], w2=d["w2"], h_q=e(n, 2 * w.F, t=torch.int8),
               h_scale=e(w.F // 16, n, t=f32), y_perm=e(n, w.D), ws=d["ws"])
    bwd = dict(dy=d["dy"], x=d["x"], prob_perm=d["pp"], row_of_slot=d["ros"], dx_perm=e(n, w.D),
               dw1=e(w.E, 2 * w.F, w.D), dw2=e(w.E, w.D, w.F), dprob_perm=e(n, t=f32),
               **{k: fwd[k] for k in ("expert_offsets", "h_q", "h_scale", "w1", "w2", "ws")})
    for fn, args in ((abi.moe_expert_ffn_ckpt, fwd), (abi.moe_expert_ffn_bwd_ckpt, bwd)):
        fn(s, **args)
        fn(s, **{k: t.reshape(-1) for k, t in args.items()})  # flat tensors have no rows to get wrong
        before = abi.moe_launch_count()
        for k, t in args.items():
            with pytest.raises(ValueError, match=f"{k} is on cpu"):
                fn(s, **{**args, k: t.cpu()})
        assert abi.moe_launch_count() == before
    torch.cuda.synchronize()
    assert abi.moe_check_device_status() == 0


def test_rows_off_the_gpu():
    from paper_2608_28511_gb300 import abi
    x = torch.randn(4, 64, device="cuda")
    q, s = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(2, 4, device="cuda")
    abi.moe_ckpt_pack(x, q, s)
    before = abi.moe_launch_count()
    for bad in ((x.cpu(), q, s), (x, q.cpu(), s), (x, q, s.cpu())):
        with pytest.raises(ValueError, match="cpu"):
            abi.moe_ckpt_pack(*bad)
        with pytest.raises(ValueError, match="cpu"):
            abi.moe_ckpt_unpack(bad[1], bad[2], bad[0])
    assert abi.moe_launch_count() == before
