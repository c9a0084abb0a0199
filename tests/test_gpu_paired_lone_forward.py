"""A lone forward (szo_model_loss) of a model whose steps run in the paired form, dense bf16 weights kept resident: the
wide rows of the paired form (weight beside eps * Zbar) must be read as such."""
import numpy as np
import pytest
import torch

from tests.fixtures import DecoderFixture

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny_gqa", "tiny"])
def test_loss_of_a_paired_model_before_and_after_steps(name):
    from paper_2406_02913_b200 import binding as B
    fx = DecoderFixture(name, seed=6, mask="random", B=3, S=20)
    om = fx.oracle_model()
    toks = torch.from_numpy(fx.batch(0)).cuda()
    S = torch.from_numpy(fx.S_init.copy()).cuda()
    m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), S, act_dtype=B.SZO_BF16, linear_mode=B.MODE_PAIRED, max_batch=3, max_seq=20)
    for step in range(3):
        want = om.loss(S.cpu().numpy(), fx.batch(0))
        assert abs(m.loss(toks).item() - want) <= 1e-3 * abs(want)          # the bf16 path's bound on the next-token loss
        out = m.zo_step(toks, 11, step, 1e-3, 1e-4).cpu().numpy()
        assert abs(out[0] - want) <= 1e-2 * abs(want)
    assert B.device_status() == 0
    m.close()
