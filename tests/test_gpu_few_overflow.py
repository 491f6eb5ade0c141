"""moe_few_tokens where silu(g) u leaves the range of bf16 or of fp32.

One expert, one product a sum: every expected value is exact up to y's own
rounding.  A value above the largest bf16 but within fp32 keeps y finite where
act is kept in more than one bf16 (fp32, and bf16 up to 32 tokens); an infinite
value gives an infinite y of the right sign at every number of tokens."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 64


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def _layer(D, dt, T):
    """g = 33/32 x_0 and u = x_1 in feature 0, nothing elsewhere; y_d = +-2^-100 silu(g) u."""
    from paper_2608_28511_gb300.layer import FewTokens
    w1 = torch.zeros(1, 2 * F, D, dtype=dt, device=DEV)
    w1[0, 0, 0] = 33 / 32
    w1[0, 64, 1] = 1.0
    w2 = torch.zeros(1, D, F, dtype=dt, device=DEV)
    w2[0, 0::2, 0] = 2.0 ** -100
    w2[0, 1::2, 0] = -2.0 ** -100
    return FewTokens(torch.zeros(1, D, dtype=dt, device=DEV), w1, w2, 1, max_tokens=T)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 1024])  # 1024: up to 8 tokens the tiles are cut along k
@pytest.mark.parametrize("T", [1, 2, 4, 8, 9, 32, 33, 128])
def test_overflow_of_the_activation(T, D, dt):
    from paper_2608_28511_gb300 import abi
    f = _layer(D, dt, T)
    big = 2.0 ** 128 * (1 - 2.0 ** -10)  # finite in fp32, rounds to infinity in bf16
    kinds = [(2.0 ** 64 * 31 / 32, 2.0 ** 64, big), (2.0 ** 64 * 31 / 32, -2.0 ** 64, -big),
             (2.0 ** 100, 2.0 ** 100, math.inf), (2.0 ** 100, -2.0 ** 100, -math.inf),
             (1.0, 1.0, (33 / 32) / (1 + math.exp(-33 / 32)))]
    for shift in range(len(kinds) if T < len(kinds) else 1):
        x = torch.zeros(T, D, dtype=dt, device=DEV)
        z = torch.empty(T, dtype=torch.float64)
        for t in range(T):
            x[t, 0], x[t, 1], z[t] = kinds[(t + shift) % len(kinds)]
        if dt == torch.bfloat16 and T > 32:  # act is one bf16
            z[z.abs() > torch.finfo(dt).max] *= math.inf
        y = f(x).double().cpu()
        assert abi.moe_check_device_status() == 0
        want = torch.stack([z * 2.0 ** -100, -z * 2.0 ** -100], 1).repeat(1, D // 2)
        same = torch.isinf(want)
        assert torch.equal(torch.isinf(y), same) and not torch.isnan(y).any(), y[:, :2]
        assert torch.equal(y[same], want[same])
        # y is rounded once (2^-9); the sigmoid of the ordinary token to a few 2^-24
        tol = 2.0 ** -8 if dt == torch.bfloat16 else 1e-5
        assert ((y - want)[~same].abs() <= tol * want[~same].abs()).all()
