"""8-bit moments whose squares are at the end of float32's range: a positive
sqrt(v) is never rounded to 0, and is 0 only where its square is."""
import numpy as np
import pytest

import optim_oracle as oo
from test_gpu_optim import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beside", [0.0, 1.0], ids=["alone", "beside 1"])
def test_small_roots_stay_positive_down_to_their_squares(beside):
    """Blocks of s = 2^-60 ... 2^-80 without a gradient, alone and with an
    element whose gradient of 1 sets the block's scale: at beta2 = 0.999 an s
    above 2^-75 has a positive square, which keeps its place among the
    denormals, and stays positive; at 2^-75 and below it is 0."""
    import torch
    import paper_2607_01164_amd as gs
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    powers = np.arange(60, 81)
    n = 32 * len(powers)
    g = np.zeros((len(powers), 32), np.float32)
    g[:, 0] = beside
    t = gs.AdamTensor.new(torch.ones(n, device="cuda"), torch.from_numpy(g.reshape(-1)).cuda(), 0.01,
                          moments=gs.GS_MOMENTS_MXFP8)
    t.v.fill_(0x38)  # 1.0
    t.v_scale.copy_(torch.from_numpy((127 - powers).astype(np.uint8)))
    gs.gs_adamw(gs.AdamPlan([t]), step=7, eps=1e-15)
    s = oo.values(host(t.v), host(t.v_scale)).reshape(-1, 32)[:, 1:]
    assert np.all(s[powers < 75] > 0) and np.all(s[powers >= 75] == 0)
    assert np.isfinite(host(t.param)).all()
