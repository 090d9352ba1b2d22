"""Host-side checks of the entry points around positions and the quantized cache: sizes, and every refusal before a launch
(the addresses are never dereferenced)."""
import ctypes

import pytest

from paper_2203_15952_amd import binding as B

INVALID, UNSUPPORTED, WORKSPACE = B.AQT_ERR_INVALID_ARG, B.AQT_ERR_UNSUPPORTED, B.AQT_ERR_WORKSPACE
ONE, BIG = 1 << 40, 1 << 44   # two addresses far apart


@pytest.fixture(scope="module")
def L():
    return B.lib()


def spec(**kw):
    d = dict(heads=4, kv_heads=2, dh=16, norm=1, eps=1e-6, rot=16, pairing=0, gamma_q=ONE, gamma_k=ONE, turns=ONE)
    d.update(kw)
    return ctypes.byref(B.aqt_qk_norm_rotate(*[d[n] for n, _ in B.aqt_qk_norm_rotate._fields_]))


def cache(**kw):
    d = dict(streams=2, capacity=128, kv_heads=2, dh=16, bits=8, data=ONE, length=ONE)
    d.update(kw)
    return ctypes.byref(B.aqt_cache(*[d[n] for n, _ in B.aqt_cache._fields_]))


BAD_SPECS = [(dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID), (dict(dh=0), INVALID),
             (dict(dh=129, rot=0), UNSUPPORTED), (dict(rot=18), INVALID), (dict(rot=3), INVALID), (dict(rot=-2), INVALID),
             (dict(turns=None), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(pairing=2), INVALID)]


@pytest.mark.parametrize("kw,status", BAD_SPECS)
def test_rotation_refuses_the_spec(L, kw, status):
    assert L.aqt_qk_norm_rotate_fwd(ONE, 2, 3, spec(**kw), None, BIG, None) == status
    assert L.aqt_qk_norm_rotate_bwd(ONE, ONE, 2, 3, spec(**kw), None, BIG, None, None, None, 0, None) == status


def test_rotation_refuses_arguments(L):
    fwd, bwd = L.aqt_qk_norm_rotate_fwd, L.aqt_qk_norm_rotate_bwd
    assert fwd(ONE, 2, 3, None, None, BIG, None) == INVALID
    assert fwd(None, 2, 3, spec(), None, BIG, None) == INVALID and fwd(ONE, 2, 3, spec(), None, None, None) == INVALID
    assert fwd(ONE, 0, 3, spec(), None, BIG, None) == INVALID and fwd(ONE, 2, 0, spec(), None, BIG, None) == INVALID
    assert fwd(ONE, 1 << 40, 1 << 40, spec(), None, BIG, None) == UNSUPPORTED
    assert fwd(ONE, 1 << 30, 1 << 21, spec(heads=1 << 20, kv_heads=1 << 20), None, BIG, None) == UNSUPPORTED
    assert fwd(ONE, 2, 3, spec(), None, ONE + 64, None) == INVALID            # overlaps, but is not, the input
    need = B.aqt_workspace_bytes(B.AQT_OP_QK_NORM_ROTATE_BWD, 6, 16, 1)
    assert need >= 2 * 16 * 4 and B.aqt_workspace_bytes(B.AQT_OP_QK_NORM_ROTATE_BWD, 6, 129, 1) == 0
    assert bwd(ONE, BIG, 2, 3, spec(), None, None, None, None, None, 0, None) == INVALID
    assert bwd(ONE, None, 2, 3, spec(), None, BIG, None, None, None, 0, None) == INVALID
    assert bwd(None, ONE, 2, 3, spec(), None, BIG, None, None, None, 0, None) == INVALID     # norm needs the input
    assert bwd(ONE, BIG, 2, 3, spec(), None, ONE, None, None, None, 0, None) == INVALID      # would overwrite the input
    assert bwd(ONE, BIG, 2, 3, spec(), None, BIG + 4, None, None, None, 0, None) == INVALID
    assert bwd(ONE, BIG, 2, 3, spec(norm=0), None, 3 * BIG, ONE, None, ONE, need, None) == INVALID    # gains without norm
    assert bwd(ONE, BIG, 2, 3, spec(), None, 3 * BIG, ONE, None, ONE, need - 1, None) == WORKSPACE
    assert bwd(ONE, BIG, 2, 3, spec(), None, 3 * BIG, None, ONE, None, need, None) == WORKSPACE
    for rot, base, turns, status in [(0, 1e4, ONE, INVALID), (3, 1e4, ONE, INVALID), (130, 1e4, ONE, UNSUPPORTED), (4, 0.0, ONE, INVALID),
                                     (4, float("nan"), ONE, INVALID), (4, float("inf"), ONE, INVALID), (4, 1e4, None, INVALID)]:
        assert L.aqt_rotation_turns(rot, base, turns, None) == status


BAD_CACHES = [(dict(streams=0), INVALID), (dict(capacity=0), INVALID), (dict(capacity=100), INVALID), (dict(capacity=-64), INVALID),
              (dict(kv_heads=0), INVALID), (dict(dh=0), INVALID), (dict(dh=129), UNSUPPORTED), (dict(bits=1), UNSUPPORTED),
              (dict(bits=9), UNSUPPORTED), (dict(streams=1 << 25), UNSUPPORTED), (dict(capacity=1 << 32), UNSUPPORTED),
              (dict(streams=1 << 24, capacity=1 << 24, kv_heads=4096), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_calls_refuse_the_shape(L, kw, status):
    c = cache(**kw)
    assert L.aqt_cache_bytes(c) == 0 and L.aqt_attention_cached_workspace_bytes(c, 1, 4) == 0
    assert L.aqt_cache_append(ONE, 1, 4, c, None, None, None) == status
    assert L.aqt_cache_read(c, 0, None, None, 1, ONE, ONE, None) == status
    assert L.aqt_attention_cached_fwd(ONE, 1, 4, c, None, -1, 0, BIG, None, ONE, BIG, None) == status
    with pytest.raises(B.AqtError):
        d = dict(streams=2, capacity=128, kv_heads=2, dh=16, bits=8) | kw
        B.KvCache(d["streams"], d["capacity"], d["kv_heads"], d["dh"], d["bits"], device="cpu")


def test_cache_calls_refuse_arguments(L):
    for bad in (dict(data=None), dict(length=None), dict(data=ONE + 8)):
        c = cache(**bad)
        assert L.aqt_cache_append(ONE, 1, 4, c, None, None, None) == INVALID
        assert L.aqt_cache_read(c, 0, None, None, 1, ONE, ONE, None) == INVALID
        assert L.aqt_attention_cached_fwd(ONE, 1, 4, c, None, -1, 0, BIG, None, ONE, BIG, None) == INVALID
    c = cache()
    app, att = L.aqt_cache_append, L.aqt_attention_cached_fwd
    assert app(None, 1, 4, c, None, None, None) == INVALID and app(ONE, 0, 4, c, None, None, None) == INVALID
    assert app(ONE, 1, 3, c, None, None, None) == INVALID and app(ONE, 1, 0, c, None, None, None) == INVALID
    assert app(ONE, 1, 4, None, None, None, None) == INVALID
    assert app(ONE, 1 << 41, 4, c, None, None, None) == UNSUPPORTED
    assert L.aqt_cache_read(c, -1, None, None, 1, ONE, ONE, None) == INVALID
    assert L.aqt_cache_read(c, 0, None, None, 0, ONE, ONE, None) == INVALID
    assert L.aqt_cache_read(c, 0, None, None, 1, None, None, None) == INVALID
    assert L.aqt_cache_read(c, 0, None, None, 1 << 41, ONE, ONE, None) == UNSUPPORTED
    assert L.aqt_cache_read(c, 0, None, None, 1 << 36, ONE, ONE, None) == UNSUPPORTED       # more workgroups than a launch has
    need = L.aqt_attention_cached_workspace_bytes(c, 1, 4)
    assert need >= 256
    assert att(None, 1, 4, c, None, -1, 0, BIG, None, ONE, need, None) == INVALID
    assert att(ONE, 1, 4, c, None, -1, 0, None, None, ONE, need, None) == INVALID
    assert att(ONE, 1, 4, c, None, -1, 0, ONE + 128, None, ONE, need, None) == INVALID      # ctx inside qkv
    assert att(ONE, 1, 6 + 1, c, None, -1, 0, BIG, None, ONE, need, None) == INVALID
    assert att(ONE, 1, 4, c, None, -1, 0, BIG, None, None, need, None) == WORKSPACE
    assert att(ONE, 1, 4, c, None, -1, 0, BIG, None, ONE, need - 1, None) == WORKSPACE
    assert att(ONE, 1 << 25, 4, c, None, -1, 0, BIG, None, ONE, BIG, None) == UNSUPPORTED
    many = cache(streams=1 << 24, kv_heads=1)                                               # 2^32 threads and more in a launch
    assert app(ONE, 1, 1, many, None, None, None) == UNSUPPORTED
    assert L.aqt_cache_read(many, 0, None, None, 1, ONE, ONE, None) == UNSUPPORTED
    assert L.aqt_attention_cached_workspace_bytes(many, 1, 1) == 0
    assert att(ONE, 1, 1, many, None, -1, 0, BIG, None, ONE, BIG, None) == UNSUPPORTED
    assert att(ONE, 1 << 14, 16, cache(streams=1 << 10, kv_heads=16, dh=8), None, -1, 0, BIG, None, ONE, BIG, None) == UNSUPPORTED
    adv = L.aqt_cache_advance
    assert adv(None, 2, 1, None, None) == INVALID and adv(ONE, 0, 1, None, None) == INVALID and adv(ONE, 2, 0, None, None) == INVALID


def test_cache_sizes(L):
    # codes of keys and values padded to 16 columns (packed values: 32), and two float32 scales per frame and head
    def nbytes(**kw):
        return L.aqt_cache_bytes(cache(data=None, length=None, **kw))
    assert nbytes(dh=64) == 2 * 2 * 128 * (2 * 64 + 8)
    assert nbytes(dh=64, bits=4) == 2 * 2 * 128 * (2 * 32 + 8)
    assert nbytes(dh=36) == 2 * 2 * 128 * (2 * 48 + 8)
    assert nbytes(dh=36, bits=4) == 2 * 2 * 128 * (24 + 32 + 8)
    assert nbytes(dh=1, bits=5) == 2 * 2 * 128 * (2 * 16 + 8)


def test_workspace_does_not_depend_on_what_a_window_hides(L):
    # one split per wavefront's share of the tiles at most, and none where the streams fill the chip by themselves
    few = L.aqt_attention_cached_workspace_bytes(cache(streams=1, capacity=1 << 20), 1, 4)
    many = L.aqt_attention_cached_workspace_bytes(cache(streams=1 << 12, capacity=1 << 10), 1, 4)
    assert few > many == 256
