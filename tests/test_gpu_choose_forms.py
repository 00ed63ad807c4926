"""The choice of experts and its gradient for numbers of experts, and distances of rows, that are no whole pieces of 16 bytes: every width of the kernels
with single loads, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import grouped_reference as ref
from tests.test_gpu_grouped import mq, scores_of, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

# (M, E, top, scores behind a row's end): one for every width of either kernel (1 lane to 64), the widest ones twice
SIZES = [(70, 7, 7, 0), (33, 15, 9, 0), (65, 31, 31, 0), (40, 63, 8, 0), (37, 65, 32, 0), (29, 127, 31, 0), (18, 128, 7, 1), (21, 201, 32, 0), (9, 256, 8, 3),
         (13, 257, 32, 0), (7, 511, 6, 0), (10, 513, 32, 0), (5, 1023, 32, 0), (3, 1024, 9, 2)]


@pytest.mark.parametrize("how", ["plain", "ties", "masked", "far", "broken"])
@pytest.mark.parametrize("M,E,top,behind", SIZES)
@pytest.mark.parametrize("renormalize", [False, True])
def test_choose(mq, M, E, top, behind, renormalize, how):  # noqa: F811
    rng = np.random.default_rng(M + 999 * E)
    s = scores_of(rng, M, E, how)
    wide = torch.full((M, E + behind), 1e30, device="cuda")   # (what stands behind a row is larger than its scores)
    wide[:, :E] = to_gpu(s)
    scores = wide[:, :E]
    ids, w, bar = ref.choose(s, top, renormalize)
    got_ids, got = mq.mq_experts_choose(scores, top, renormalize=renormalize)
    assert np.array_equal(got_ids.cpu().numpy(), ids)
    weight = got.cpu().double().numpy()
    assert np.array_equal(np.isnan(weight), np.isnan(w))
    ok = ~np.isnan(w)
    assert (np.abs(weight - w)[ok] <= bar[ok]).all()
    if how == "broken":
        return
    dw = rng.standard_normal((M, top)).astype(np.float32)
    dw[ids < 0] = np.nan   # of no choice: not looked at
    room = torch.full((M * E + 8,), 7.0, device="cuda")
    ds = mq.mq_experts_choose_bwd(scores, got_ids, got, to_gpu(dw), renormalize=renormalize, dscores=room[4:4 + M * E].view(M, E))
    want, far = ref.choose_bwd(s, ids, got.cpu().numpy(), dw, renormalize)
    assert (np.abs(ds.cpu().double().numpy() - want) <= far).all()
    assert (room[:4] == 7).all() and (room[4 + M * E:] == 7).all()
