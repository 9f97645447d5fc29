"""Refusals and host arithmetic of the operators on cached context; no GPU is touched.  And the 64-bit reference against hand-worked values."""
import numpy as np
import pytest

import context_ref as ref
import oracle
from paper_2409_13761_b200 import kdn as K

D128 = K.pool_desc(4, 2, 128, 16, 64)
G64 = K.KDN_CODEC_INT4_G64


def chunk(desc=D128, T=20, codec=G64, data=0x10000, mem=0, base=0):
    return K.Chunk(data, K.kdn_chunk_bytes(desc, T, codec), T, codec, mem, base)


def attend(reqs=None, desc=D128, layer=0, **kw):
    io = dict(q=0x20000, out=0x30000, n_q_heads=8, scale=0.1, rope_theta=1e4)
    io.update(kw)
    return K.kdn_validate_attend(desc, layer, [K.AttendReq(1, 100, [chunk(desc)], [0])] if reqs is None else reqs, **io)


def test_attend_refusals():
    ok, bad, uns, al = K.KDN_OK, K.KDN_E_INVAL, K.KDN_E_UNSUPPORTED, K.KDN_E_ALIGN
    assert attend() == ok and attend([]) == ok
    assert attend(layer=4) == bad and attend(layer=-1) == bad
    assert attend(q=0) == bad and attend(out=0) == bad and attend(q=0x20008) == al and attend(out=0x30002) == al and attend(lse=2) == al
    assert attend(n_q_heads=0) == bad and attend(n_q_heads=7) == bad and attend(n_q_heads=-2) == bad
    assert attend(q_stride=1023) == bad and attend(out_stride=8) == bad and attend(q_stride=1028) == al
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e300):
        assert attend(scale=scale) == bad
    assert attend(rope_style=1) == uns
    assert attend(rope_theta=0.0) == ok                                                   # nothing is rotated
    moved = [K.AttendReq(1, 100, [chunk(base=3)], [0])]
    assert attend(moved) == ok
    for theta in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(moved, rope_theta=theta) == bad
    for codec in (0, 1, 3, 5, 6):
        assert attend([K.AttendReq(1, 100, [chunk(codec=codec)], [0])]) == uns
    assert attend([K.AttendReq(1, 100, [chunk(codec=7)], [0])]) == bad
    assert attend([K.AttendReq(1, 100, [chunk(codec=K.KDN_CODEC_INT4_KC64)], [5])]) == ok   # no rule on where the part stands
    assert attend([K.AttendReq(1, 100, [chunk(mem=1)], [0])]) == uns
    assert attend([K.AttendReq(1, 100, [chunk(data=0)], [0])]) == bad
    assert attend([K.AttendReq(1, 100, [chunk(data=0x10008)], [0])]) == al
    c = chunk()
    c.bytes -= 1
    assert attend([K.AttendReq(1, 100, [c], [0])]) == K.KDN_E_SHAPE
    assert attend([K.AttendReq(-1, 100, [], [])]) == bad
    assert attend([K.AttendReq(1, -1, [], [])]) == bad and attend([K.AttendReq(1, 1 << 40, [], [])]) == bad
    assert attend([K.AttendReq(1, 0, [chunk()], [-1])]) == bad and attend([K.AttendReq(1, 0, [chunk()], [1 << 40])]) == bad
    assert attend([K.AttendReq(1, 0, [chunk(base=-1)], [0])]) == bad
    assert attend([K.AttendReq(0, 0, [chunk()], [0])], q=0, out=0) == ok                  # no rows: nothing to write
    for dim, want in ((64, ok), (128, ok), (192, uns), (256, uns)):
        d = K.pool_desc(1, 2, dim, 16, 64)
        assert attend(desc=d) == want
    with pytest.raises(ValueError):
        K.attend_array([K.AttendReq(1, 0, [chunk()], [])])
    arr = K.attend_array([K.AttendReq(1, 0, [chunk()], [0])])
    assert K.lib.kdn_validate_attend(None, 0, arr, 1, None) == bad
    io = K.kdn_attend_io(0x20000, 0x30000, 0, 1024, 1024, 8, 0, 1e4, 0.1, 0, 0)
    assert K.lib.kdn_validate_attend(D128, 0, None, 1, io) == bad
    assert K.lib.kdn_validate_attend(D128, 0, arr, -1, io) == bad
    assert K.lib.kdn_validate_attend(D128, 0, arr, 1, io) == ok
    arr[0].parts = None
    assert K.lib.kdn_validate_attend(D128, 0, arr, 1, io) == bad
    assert attend([K.AttendReq(1 << 30, 0, [], [])]) == uns                               # rows x heads past 31 bits


def weigh(reqs=None, desc=D128, layer=0, **kw):
    io = dict(q=0x20000, n_q_heads=8, scale=0.1)
    io.update(kw)
    return K.kdn_validate_weigh(desc, layer, [K.WeighReq(0x1000, 4, 60, 1, 59, 0x4000, 60)] if reqs is None else reqs, **io)


def test_weigh_refusals():
    ok, bad, uns, al = K.KDN_OK, K.KDN_E_INVAL, K.KDN_E_UNSUPPORTED, K.KDN_E_ALIGN
    R = K.WeighReq
    assert weigh() == ok and weigh([]) == ok
    assert weigh(layer=4) == bad and weigh(q=0) == bad and weigh(q=0x20004) == al and weigh(lse=6) == al
    assert weigh(lse_given=True) == bad and weigh(lse_given=True, lse=0x8000) == ok
    assert weigh(n_q_heads=3) == bad and weigh(q_stride=100) == bad and weigh(q_stride=1025) == al
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert weigh(scale=scale) == bad
    assert weigh([R(0x1000, 4, 64, 1, 0, 0x4000, 64)]) == ok
    assert weigh([R(0x1000, 4, 65, 1, 0, 0x4000, 65)]) == K.KDN_E_RANGE
    assert weigh([R(0, 4, 60, 1, 0, 0x4000, 60)]) == bad and weigh([R(0x1000, 4, 60, 1, 0, 0, 60)]) == bad
    assert weigh([R(0x1000, 4, 60, 1, 0, 0x4000, 59)]) == bad and weigh([R(0x1000, 4, 60, 1, 0, 0x4002, 60)]) == al
    assert weigh([R(0x1000, 4, -1, 1, 0, 0x4000, 60)]) == bad and weigh([R(0x1000, 4, 60, -1, 0, 0x4000, 60)]) == bad
    assert weigh([R(0x1000, 4, 60, 1, -1, 0x4000, 60)]) == bad and weigh([R(0x1000, -4, 0, 1, 0, 0x4000, 60)]) == bad
    assert weigh([R(0, 0, 0, 3, 0, 0, 0)]) == ok                                          # a context of no tokens
    assert weigh(desc=K.pool_desc(1, 2, 96, 16, 64)) == uns


def evict(**kw):
    r = dict(weights=0x1000, n_rows=3, n_tokens=50, row_stride=50, n_keep=20, n_first=4, n_last=8, keep=0x2000, kept=0x3000, kept_stride=20)
    r.update(kw)
    return K.kdn_validate_evict([K.EvictReq(**r)])


def test_evict_refusals():
    ok, bad, rng, al = K.KDN_OK, K.KDN_E_INVAL, K.KDN_E_RANGE, K.KDN_E_ALIGN
    assert evict() == ok and K.kdn_validate_evict([]) == ok
    assert evict(n_keep=50, kept_stride=50) == ok and evict(n_keep=51, kept_stride=51) == rng
    assert evict(n_first=12) == ok and evict(n_first=13) == rng and evict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1) == rng
    for name in ("n_tokens", "n_keep", "n_first", "n_last"):
        assert evict(**{name: -1}) == bad
    assert evict(n_rows=0) == bad and evict(weights=0) == bad and evict(keep=0) == bad and evict(kept=0, kept_stride=0) == ok
    assert evict(row_stride=49) == bad and evict(kept_stride=19) == bad
    assert evict(weights=0x1002) == al and evict(keep=0x2001) == al and evict(kept=0x3002) == al
    assert evict(n_tokens=0, n_keep=0, n_first=0, n_last=0, weights=0, keep=0) == ok
    assert evict(n_keep=0, n_first=0, n_last=0, keep=0) == ok
    assert K.kdn_evict_workspace([K.EvictReq(0x1000, 3, 50, 50, 20, 4, 8, 0x2000)]) >= 200
    with pytest.raises(K.KdnError):
        K.kdn_evict_workspace([K.EvictReq(0x1000, 3, 50, 50, 60, 4, 8, 0x2000)])


def test_sizes_past_the_limits_are_refused():
    uns, most = K.KDN_E_UNSUPPORTED, 1 << 28
    small = K.pool_desc(1, 1, 64, 16, 64)
    assert attend([K.AttendReq(1, 100, [chunk(small, T=most)], [0])], desc=small) == K.KDN_OK
    assert attend([K.AttendReq(1, 100, [chunk(small, T=most + 1)], [0])], desc=small) == uns
    blocks = most // 16 + 1
    assert weigh([K.WeighReq(0x1000, blocks, most, 1, 59, 0x4000, most)]) == K.KDN_OK
    assert weigh([K.WeighReq(0x1000, blocks, most + 1, 1, 59, 0x4000, most + 1)]) == uns
    assert weigh([K.WeighReq(0x1000, blocks, most, 1, 59, 0x4000, most)] * 200) == uns         # more tiles than 31 bits number
    assert weigh([K.WeighReq(0x1000, blocks, most, 1 << 20, 59, 0x4000, most)]) == uns
    assert evict(n_tokens=most, row_stride=most) == K.KDN_OK and evict(n_rows=most) == K.KDN_OK
    assert evict(n_tokens=most + 1, row_stride=most + 1) == uns and evict(n_rows=most + 1) == uns


def test_scales_that_fp32_does_not_hold_are_refused():
    """The kernels work in powers of two: what they multiply by is scale * log2(e) in fp32."""
    for scale in (1e-46, 2.4e38, 3.4e38, 1e-300):
        assert attend(scale=scale) == K.KDN_E_INVAL and weigh(scale=scale) == K.KDN_E_INVAL
    for scale in (1e-38, 1.0, 2.3e38):
        assert attend(scale=scale) == K.KDN_OK and weigh(scale=scale) == K.KDN_OK


def test_calls_without_a_context_are_refused():
    arr = K.attend_array([])
    assert K.lib.kdn_attend(None, 0, 0, arr, 0, None, None) == K.KDN_E_INVAL
    assert K.lib.kdn_weigh(None, 0, 0, None, 0, None, None) == K.KDN_E_INVAL
    assert K.lib.kdn_evict(None, None, 0, None, 0, None) == K.KDN_E_INVAL
    assert K.lib.kdn_attend_workspace(None, 0, arr, 0, 8, None) == K.KDN_E_INVAL
    assert K.lib.kdn_evict_workspace(None, 0, None) == K.KDN_E_INVAL
    with pytest.raises(K.KdnError):
        K.kdn_attend(None, 0, 0, [], q=0, out=0, n_q_heads=1, scale=1.0)


# ---------------------------------------------------------------------- the reference itself --

def test_reference_attention_by_hand():
    # two tokens, one head of two channels: scores ln 3 and 0, so weights 3/4 and 1/4
    k = np.array([[[np.log(3.0), 0.0]], [[0.0, 5.0]]])
    v = np.array([[[4.0, 8.0]], [[0.0, -8.0]]])
    q = np.array([[[1.0, 0.0]]])
    out, lse, mass, reach = ref.attend(q, [(k, v, 0, 0)], 5, 1.0, 1e4)
    assert np.allclose(out, [[[3.0, 4.0]]]) and np.allclose(lse, np.log(4.0)) and np.allclose(mass, [[[3.0, 8.0]]])
    out, lse, _, _ = ref.attend(q, [(k, v, 0, 0)], 0, 1.0, 1e4)                            # sees the first token only
    assert np.allclose(out, [[[4.0, 8.0]]]) and np.allclose(lse, np.log(3.0))
    out, lse, _, _ = ref.attend(q, [(k, v, 3, 3)], 2, 1.0, 1e4)                            # sees nothing
    assert (out == 0).all() and np.isneginf(lse).all()
    # a quarter turn: with two channels the angle is the shift itself
    assert np.allclose(ref.rotate(np.array([1.0, 0.0]), 1, 1e4), [np.cos(1.0), np.sin(1.0)])


def test_reference_decode_is_the_oracles():
    rng = np.random.default_rng(1)
    L, H, D, T = 2, 3, 64, 70
    pool = ref.bits(rng.standard_normal((L, 2, 5, 16, H, D)))
    table = np.arange(5, dtype=np.int32)
    for codec in (oracle.INT4_G64, oracle.INT4_KC64):
        data = oracle.store(pool, table, 0, T, codec)
        back = pool.copy()
        oracle.retrieve(back, table, 0, T, codec, data)
        for layer in range(L):
            for kv, x in enumerate(ref.decode(data, L, H, D, T, codec == oracle.INT4_KC64, layer)):
                want = back[layer, kv].reshape(-1, H, D)[:T]
                assert np.array_equal(ref.bits(x.astype(np.float32)), want)


def test_reference_weights_and_ranking_by_hand():
    k = np.array([[[np.log(2.0)]], [[0.0]], [[np.log(5.0)]]])
    q = np.ones((2, 1, 1))
    add, lse, _ = ref.weigh(q, k, 1, 1.0)
    assert np.allclose(lse[:, 0], [np.log(3.0), np.log(8.0)])
    assert np.allclose(add[0], [2 / 3 + 2 / 8, 1 / 3 + 1 / 8, 5 / 8])
    assert ref.evict(np.array([[1, 5, 5, 0, 9, 5.0]]), 3, 0, 0).tolist() == [1, 2, 4]
    assert ref.evict(np.array([[1, 5, 5, 0, 9, 5.0]]), 3, 1, 1).tolist() == [0, 4, 5]
    assert ref.evict(np.array([[np.nan, -np.inf, 1.0]]), 2, 0, 0).tolist() == [0, 2]
