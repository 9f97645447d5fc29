"""The operators on cached context at their edges: workspaces that hold what an earlier call left, key scales far from 1 or zero, huge and infinite
scales in tokens that only some rows see, log-sum-exps far below the scores.  Against the same in 64 bits."""
import numpy as np
import pytest
import torch

import context_ref as ref
import oracle
from test_gpu_attend import Case as AttendCase, make as make_attend
from test_gpu_weigh import Case as WeighCase

pytestmark = pytest.mark.gpu
G64, KC64 = oracle.INT4_G64, oracle.INT4_KC64


# --------------------------------------------------------------------------- what a workspace holds --

def weigh_on(c, space):
    """The call on a workspace of the caller's."""
    K, dev = c.dev.K, c.dev
    assert K.kdn_weigh_workspace(dev.ctx, dev.pool_id, c.recs, c.Hq, False) <= space.numel()
    for a, b in zip(c.acc, c.acc0):
        a.copy_(torch.from_numpy(b))
    torch.cuda.synchronize()
    K.kdn_weigh(dev.ctx, dev.pool_id, c.layer, c.recs, q=c.q.data_ptr(), q_stride=c.q.stride(0), lse=c.lse.data_ptr(), n_q_heads=c.Hq, scale=c.scale,
                workspace=space.data_ptr(), workspace_bytes=space.numel(), stream=dev.stream.cuda_stream)
    return c


@pytest.mark.parametrize("n_q", [1, 4, 40])
@pytest.mark.parametrize("H,tokens", [(1, 288), (1, 1050), (1, 33), (2, 160), (2, 1000), (4, 97), (3, 2000)])
def test_weigh_reads_nothing_that_the_workspace_held(H, tokens, n_q):
    """Counts of tiles that eight warps a CTA do not divide.  The workspace holds NaN, then what a call over a longer context with louder queries left; both
    calls give the same bits."""
    rng = np.random.default_rng(H + tokens + n_q)
    reqs = [(n_q, tokens - 1, tokens)]
    c = WeighCase(rng, H, 128, 4, 16, reqs)
    big = WeighCase(rng, H, 128, 4, 16, [(n_q, 20000, 20000)], q_gain=30.0)
    try:
        big.call()
        assert big.dev.sync() == 0
        nan = torch.full_like(big.space, 0xFF)
        first = weigh_on(c, nan).check()
        first = first.acc[0].clone(), first.lse.clone()
        weigh_on(c, big.space).check()
        assert torch.equal(first[0], c.acc[0]) and torch.equal(first[1], c.lse)
    finally:
        c.close()
        big.close()


def test_weigh_of_ragged_requests_reads_nothing_that_the_workspace_held():
    """More requests than travel as launch parameters, some of one tile, some of none."""
    rng = np.random.default_rng(5)
    c = WeighCase(rng, 1, 64, 2, 16, [(int(rng.integers(1, 9)), int(rng.integers(0, 200)), int(rng.integers(0, 200))) for _ in range(21)])
    try:
        need = c.dev.K.kdn_weigh_workspace(c.dev.ctx, c.dev.pool_id, c.recs, c.Hq, False)
        weigh_on(c, torch.full((need,), 0xFF, dtype=torch.uint8, device=c.dev.dev)).check()
    finally:
        c.close()


@pytest.mark.parametrize("codec", [G64, KC64])
@pytest.mark.parametrize("n_q", [1, 3, 15])
def test_attend_reads_nothing_that_the_workspace_held(codec, n_q):
    for H in (1, 2, 8):
        dev = make_attend(H, 128)
        try:
            rng = np.random.default_rng(H + n_q)
            c = AttendCase(dev, rng, [(n_q, 700, [(333, codec, 9, 0), (290, codec, 0, 333)]), (1, 40, [(70, codec, 0, 0)])], 4)
            need = dev.K.kdn_attend_workspace(dev.ctx, dev.pool_id, c.recs, c.Hq)
            c.call(workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device=dev.dev)).check()
        finally:
            dev.close()
