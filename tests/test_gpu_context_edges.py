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


# --------------------------------------------------------------------------- key scales far from 1 --

def edit_scales(c, j, D, H, T, codec, keys=None, values=None):
    """Part j of the first request: `keys` and `values` change the scales of the layer that is attended to, in place: [T][H][D/64], or keys in channel
    groups [groups][H][D]."""
    L, layer = c.dev.shape.n_layers, c.layer
    buf = c.keep[j]
    raw = buf.cpu().numpy()
    scales = raw[L * 2 * (T * H * D // 2):].view(np.float32)
    row = T * H * (D // 64)
    per_key = -(-T // 64) * H * D if codec == KC64 else row
    k0 = layer * (per_key + row)
    k = scales[k0:k0 + per_key].reshape((-1, H, D) if codec == KC64 else (T, H, D // 64))
    v = scales[k0 + per_key:k0 + per_key + row].reshape(T, H, D // 64)
    if keys is not None:
        keys(k)
    if values is not None:
        values(v)
    buf.copy_(torch.from_numpy(raw))
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        planes = ref.decode(raw, L, H, D, T, codec == KC64, layer)
    old = c.refs[0][3][j]
    c.refs[0][3][j] = (planes[0], planes[1], old[2], old[3])


GROUPS = {
    "zero first": [0.0, 1.0, 1.0, 1.0],
    "zero in the middle": [1.0, 0.0, 0.0, 1.0],
    "zero last": [1.0, 1.0, 1.0, 0.0],
    "all zero": [0.0, 0.0, 0.0, 0.0],
    "tiny and back": [1.0, 1e-30, 1.0, 1e-10],
    "smallest normal and back": [1.0, 2.0 ** -126 / 0.02, 0.0, 1.0],
    "up": [1e-30, 1e-20, 1e-10, 1.0],
    "huge and back": [1.0, 1e30, 1e-30, 1.0],
    "down": [1e30, 1e10, 1.0, 1e-30],
}


@pytest.mark.parametrize("what", GROUPS)
@pytest.mark.parametrize("n_q", [1, 10, 11, 40])
@pytest.mark.parametrize("D,H", [(64, 1), (64, 8), (128, 2), (128, 8)])
def test_channel_groups_of_zero_and_far_scales(what, n_q, D, H):
    """Keys in channel groups: a factor on all scales of a group of 64 tokens, for the even heads (the odd ones stay as they are)."""
    T, codec = 64 * 3 + 50, KC64
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(D + H + n_q)
        c = AttendCase(dev, rng, [(n_q, 500, [(T, codec, 7, 0), (T, codec, T, T)])], 4)

        def keys(k):
            k[:, ::2] *= np.array(GROUPS[what], dtype=np.float32)[:, None, None]

        for j in range(2):
            edit_scales(c, j, D, H, T, codec, keys=keys)
        c.call().check()
    finally:
        dev.close()


@pytest.mark.parametrize("n_q", [1, 10, 11])
def test_a_chunk_of_keys_that_were_never_written(n_q):
    """Stored by the library from a pool that holds zeros for 64 tokens and more."""
    H, D, T = 2, 128, 300
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(3)
        pool = ref.bits(rng.standard_normal((2, 2, 19, 16, H, D)))
        pool[:, 0, 3:14] = 0
        data = oracle.store(pool, np.arange(19, dtype=np.int32), 0, T, KC64)
        c = AttendCase(dev, rng, [(n_q, 400, [(T, KC64, 0, 0)])], 4)
        c.keep[0].copy_(torch.from_numpy(data))
        k, v = ref.decode(data, 2, H, D, T, True, c.layer)
        assert (k[64:192] == 0).all()
        c.refs[0][3][0] = (k, v, 0, 0)
        c.call().check()
    finally:
        dev.close()


# ----------------------------------------------------------------- tokens that only some rows see --

@pytest.mark.parametrize("value", [float("inf"), 1e20, 3e38, 1e4])
@pytest.mark.parametrize("n_q,g,H", [(2, 4, 2), (2, 4, 8), (2, 1, 16), (3, 16, 2), (40, 4, 2), (300, 1, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_tokens_that_later_rows_see_do_not_matter(value, n_q, g, H, D):
    """The key scales of the last token that is seen at all, by the last new token only, are huge or infinite: the rows before it keep their bits."""
    T, codec = 80 + n_q + 100, G64
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(n_q + D)
        c = AttendCase(dev, rng, [(n_q, 80, [(T, codec, 0, 0)])], g).call().check()
        want, want_lse = c.out.clone(), c.lse.clone()

        def keys(k):
            k[80 + n_q - 1] = value

        edit_scales(c, 0, D, H, T, codec, keys=keys)
        c.call()
        assert dev.sync() == 0
        assert torch.equal(c.out[:-1], want[:-1]) and torch.equal(c.lse[:-1], want_lse[:-1])
        if value < 1e30:                                                      # (products with 3e38 pass what 32 bits hold)
            c.check()
    finally:
        dev.close()


@pytest.mark.parametrize("value", [float("inf"), 1e4])
@pytest.mark.parametrize("n_q", [2, 5])
def test_a_row_rounds_by_what_it_sees_itself(value, n_q):
    """The same with so many requests (over one chunk) that each is gone through tile by tile in one place; a token of the last of three tiles has some
    rows move their reference but not the others."""
    H, D, codec, seen = 8, 64, G64, 32 * 3 - 10
    dev = make_attend(H, D, L=1)
    try:
        rng = np.random.default_rng(n_q)
        c = AttendCase(dev, rng, [(n_q, seen - n_q, [(seen, codec, 0, 0)]) for _ in range(296)], 4, layer=0)
        for r in c.recs:
            r.parts = c.recs[0].parts
        c.call()
        assert dev.sync() == 0
        want, want_lse = c.out.clone(), c.lse.clone()

        def keys(k):
            k[seen - 1] = value

        edit_scales(c, 0, D, H, seen, codec, keys=keys)
        c.call()
        assert dev.sync() == 0
        before = torch.arange(c.rows, device=dev.dev) % n_q != n_q - 1
        assert torch.equal(c.out[before], want[before]) and torch.equal(c.lse[before], want_lse[before])
        assert not torch.equal(c.lse[~before], want_lse[~before])
    finally:
        dev.close()


@pytest.mark.parametrize("n_q,g", [(10, 4), (33, 4), (200, 1)])
@pytest.mark.parametrize("D,turn", [(64, 0), (128, 0), (128, 9)])
def test_each_row_has_the_precision_of_what_it_sees(n_q, g, D, turn):
    """Key scales that grow from token to token, so that a row's largest score is far below those of the tile's other rows."""
    H, T, codec = 2, 30 + n_q, G64
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(n_q)
        c = AttendCase(dev, rng, [(n_q, 30, [(T, codec, turn, 0)])], g)

        def keys(k):
            k[30:] *= (8.0 ** np.minimum(np.arange(n_q), 30))[:, None, None].astype(np.float32)

        edit_scales(c, 0, D, H, T, codec, keys=keys)
        c.call().check()
    finally:
        dev.close()


@pytest.mark.parametrize("n_q", [10, 11, 70])
@pytest.mark.parametrize("D,turn", [(64, 5), (128, 0), (128, 5)])
def test_key_scales_of_many_magnitudes(n_q, D, turn):
    """Tokens and groups of channels over eight orders of magnitude, zero among them; parts of one and of many magnitudes in turn."""
    H, T, codec = 2, 333, G64
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(n_q + D)
        c = AttendCase(dev, rng, [(n_q, 1000, [(T, codec, turn, 0), (T, codec, T, T), (T, codec, 2 * T + turn, 2 * T)])], 4)

        def keys(k):
            k *= (10.0 ** rng.uniform(-8, 0, k.shape)).astype(np.float32)
            k[rng.random(T) < 0.1] = 0.0

        edit_scales(c, 1, D, H, T, codec, keys=keys)
        edit_scales(c, 2, D, H, T, codec, keys=keys)
        c.call().check()
    finally:
        dev.close()


# ------------------------------------------------------------------------------------ huge scores --

@pytest.mark.parametrize("gain", [1e6, 1e12, 1e25])
@pytest.mark.parametrize("n_q", [1, 40])
def test_weigh_with_huge_scores(gain, n_q):
    """The log-sum-exp of scores so large that one step of them in 32 bits is more than any weight's exponent (so that of the weights only this is sure:
    they are numbers).  Bounds as for other scores: 136 * 2^-24 of sum |q k| for the sums, fp32's own step for the result."""
    rng = np.random.default_rng(6)
    c = WeighCase(rng, 2, 128, 4, 16, [(n_q, 300, 300)], q_gain=gain)
    try:
        c.call()
        assert c.dev.sync() == 0
        k = c.keys[c.tables[0][np.arange(300) // 16], np.arange(300) % 16]
        add, want, reach = ref.weigh(c.q64, k, 300, c.scale)
        assert (np.abs(c.lse.cpu().numpy().astype(np.float64) - want) <= 2.0 ** -16.9 * reach + 2.0 ** -18 + 2.0 ** -22 * np.abs(want)).all()
        assert not torch.isnan(c.acc[0]).any()
    finally:
        c.close()


@pytest.mark.parametrize("gain", [1e6, 1e12, 1e25])
@pytest.mark.parametrize("codec", [G64, KC64])
@pytest.mark.parametrize("n_q", [1, 11, 70])
def test_attend_with_huge_scores(gain, codec, n_q):
    """One row's queries are huge, the others' are not: those keep their bits."""
    dev = make_attend(2, 128)
    try:
        rng = np.random.default_rng(7)
        c = AttendCase(dev, rng, [(n_q, 400, [(200, codec, 7, 0), (150, codec, 0, 200)])], 4).call().check()
        want, want_lse = c.out.clone(), c.lse.clone()
        c.q[n_q // 2, 5] *= gain
        c.q64[n_q // 2, 5] = c.q[n_q // 2, 5].double().cpu().numpy()
        c.call().check()
        assert torch.isfinite(c.out).all() and torch.isfinite(c.lse).all()
        rest = torch.ones_like(c.lse, dtype=torch.bool)
        rest[n_q // 2, 5] = False
        assert torch.equal(c.out[rest], want[rest]) and torch.equal(c.lse[rest], want_lse[rest])
    finally:
        dev.close()


@pytest.mark.parametrize("codec", [G64, KC64])
@pytest.mark.parametrize("n_q", [1, 11, 70])
def test_scores_past_the_range_of_fp32(codec, n_q):
    """A row whose scores are infinite in 32 bits is NaN, not one that saw nothing; the others keep their bits."""
    dev = make_attend(2, 128)
    try:
        rng = np.random.default_rng(7)
        c = AttendCase(dev, rng, [(n_q, 400, [(200, codec, 7, 0), (150, codec, 0, 200)])], 4).call().check()
        want, want_lse = c.out.clone(), c.lse.clone()
        c.q[n_q // 2, 5] = torch.sign(c.q[n_q // 2, 5].float()) * 1e38
        c.call()
        assert dev.sync() == 0
        assert torch.isnan(c.out[n_q // 2, 5]).all() and torch.isnan(c.lse[n_q // 2, 5])
        rest = torch.ones_like(c.lse, dtype=torch.bool)
        rest[n_q // 2, 5] = False
        assert torch.equal(c.out[rest], want[rest]) and torch.equal(c.lse[rest], want_lse[rest])
    finally:
        dev.close()


# ------------------------------------------------------------------------------- NaN that is seen --

@pytest.mark.parametrize("codec", [G64, KC64])
@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("T", [20, 64, 200])
def test_nan_in_a_value_shows_however_small_its_weight(codec, n_q, T):
    """A token whose weight is below what fp32 holds has a NaN for a value scale: the rows that see it are NaN, their lse is not."""
    H, D, bad = 2, 128, 5
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(T)
        c = AttendCase(dev, rng, [(n_q, T + 5, [(T, codec, 0, 0)])], 4, q_gain=400.0)
        raw = c.keep[0].cpu().numpy()
        row = H * D // 2
        at = 2 * c.layer * T * row + bad * row
        raw[at:at + row] = 0                                                  # a key of zeros: its score is 0, the largest some hundreds
        c.keep[0].copy_(torch.from_numpy(raw))
        edit_scales(c, 0, D, H, T, codec)
        c.call().check()
        assert (c.lse > 100.0).all()                                          # e^-100 is 2^-144
        want_lse = c.lse.clone()

        def values(v):
            v[bad] = np.nan

        edit_scales(c, 0, D, H, T, codec, values=values)
        c.call()
        assert dev.sync() == 0
        assert torch.isnan(c.out).all() and torch.equal(c.lse, want_lse)
    finally:
        dev.close()


@pytest.mark.parametrize("codec", [G64, KC64])
@pytest.mark.parametrize("n_q", [8, 40])
@pytest.mark.parametrize("plane", [0, 1])
def test_infinities_that_were_stored(codec, n_q, plane):
    """An infinite key or value leaves an infinite scale and zero codes in a chunk, whose product is no number: rows that see it are NaN, the others keep their bits."""
    H, D, T, bad = 2, 128, 200, 64                                            # (keys in channel groups: the first token of a group)
    dev = make_attend(H, D)
    try:
        rng = np.random.default_rng(12)
        x = rng.standard_normal((2, 2, 13, 16, H, D)).astype(np.float32)
        c = AttendCase(dev, rng, [(n_q, bad - 4, [(T, codec, 0, 0)])], 4)

        def put(y):
            data = oracle.store(ref.bits(y), np.arange(13, dtype=np.int32), 0, T, codec)
            c.keep[0].copy_(torch.from_numpy(data))
            with np.errstate(invalid="ignore"):
                k, v = ref.decode(data, 2, H, D, T, codec == KC64, c.layer)
            c.refs[0][3][0] = (k, v, 0, 0)
            c.call()
            return np.isnan((k, v)[plane][bad]).any()

        assert not put(x)
        c.check()
        want, want_lse = c.out.clone(), c.lse.clone()
        x[c.layer, plane, bad // 16, bad % 16, :, 5] = np.inf
        assert put(x)
        assert dev.sync() == 0
        assert torch.equal(c.out[:4], want[:4]) and torch.equal(c.lse[:4], want_lse[:4])
        # a key: the row; a value: the channels of its group of 64
        assert torch.isnan(c.out[4:, :, :64]).all()
        assert torch.isnan(c.lse[4:]).all() if plane == 0 else torch.isfinite(c.lse).all()
    finally:
        dev.close()


# --------------------------------------------------------------- a given lse far below the scores --

@pytest.mark.parametrize("below", [60.0, 88.5, 89.0, 100.0, 1000.0])
def test_given_lse_far_below_the_scores(below):
    """Weights near and past what fp32 holds, from each place of a full block of 128 rows in turn.  A power's argument of up to 2^10.6 is rounded twice in 32 bits,
    2^-14 of the result at most, and the power itself to 2^-21."""
    rng = np.random.default_rng(8)
    H = 8
    c = WeighCase(rng, H, 64, 1, 16, [(128, 400, 256)], q_gain=1e-3)
    try:
        k = c.keys[c.tables[0][np.arange(256) // 16], np.arange(256) % 16]
        score = c.scale * np.einsum("rhd,thd->rht", c.q64, k)
        for first in range(0, 128, H):
            lse = np.full((128, H), np.float32(np.log(256.0)))
            odd = [first + h for h in range(H)]                               # a row for each head
            lse[odd, range(H)] = -below
            c.lse.copy_(torch.from_numpy(lse))
            c.acc[0].copy_(torch.from_numpy(c.acc0[0]))
            c.call(given=True)
            assert c.dev.sync() == 0
            with np.errstate(over="ignore"):
                want = np.exp(score - lse.astype(np.float64)[:, :, None]).sum(0) + c.acc0[0][:, :256]
            got = c.acc[0].cpu().numpy()[:, :256].astype(np.float64)
            past = want > np.finfo(np.float32).max
            assert (past == (below > 88.8)).all()
            assert (got[past] == np.inf).all(), got[past]
            assert (np.abs(got[~past] - want[~past]) <= 2.0 ** -13 * want[~past]).all()
    finally:
        c.close()


# -------------------------------------------------------------------------------------- bookkeeping --

def test_a_destroyed_context_leaves_no_pools():
    """Row strides that are left out go by the pools of the context at hand."""
    dev = make_attend(2, 64)
    K, at = dev.K, dev.ctx.value
    assert K._head_dim(dev.ctx, dev.pool_id) == 64
    dev.close()
    assert not [k for k in K._pool_dims if k[0] == at]
