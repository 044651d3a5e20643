"""Wild segment offsets of the bidirectional attention: their differences pass 2^31."""
import numpy as np
import pytest
import torch

from tests.helpers import cuda, i32

pytestmark = pytest.mark.gpu

S = pytest.importorskip("paper_2607_14557_gb300.seer")


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [-2 ** 31, -2 ** 31 + 6, 2 ** 31 - 1, -1])
def test_a_wild_offset_costs_its_own_segments_alone(dt, bad):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    S.seer_check_device()
    H, dh, T = 2, 128, 300
    gen = torch.Generator(device=cuda()).manual_seed(1)
    x = torch.randn(T, 3 * H * dh, device=cuda(), generator=gen).to({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dt])
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device=cuda())
    outs = []
    for cu in ([0, 7, bad, 9, 9, 300], [0, 7, 9, 9, 9, 300]):
        o = torch.full((T, H * dh), 5.0, dtype=x.dtype, device=cuda())
        S.seer_attention(x, o, dt, i32(cu), None, 5, T, H, dh, ws, ws.numel())
        outs.append((o.double().cpu().numpy(), S.seer_check_device()))
    (got, code), (ref, fine) = outs
    assert code == 2 and fine == 0
    keep = np.r_[0:7, 9:300]
    if dt == "f32":                                         # its blocks find their segment by a search that needs ascending offsets
        keep = np.r_[0:0]
    assert (np.abs(got[keep] - ref[keep]) <= 2.0 ** -7 * np.abs(ref[keep]) + 2.0 ** -9).all()
    assert (got[7:9] == 5.0).all()
