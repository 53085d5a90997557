"""Cross attention and the cache held in 8 bits without a GPU: layout, bookkeeping and refusals (plan-only caches)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2511_16047_b200 import binding as B
from paper_2511_16047_b200 import synth

A = 1 << 20


def _plan(sides=(1, 2, 3), policies=((1, 1, False),), heads=4, head_dim=64, rows=2, flags=0, **kw):
    d, keep = B.make_desc(len(policies), heads, head_dim, rows, sides, policies, flags=B.FLAG_PLAN_ONLY | flags, **kw)
    return B.amskv_cache_create(d)


def _code(fn, *a, **kw):
    with pytest.raises(B.AmskvError) as e:
        fn(*a, **kw)
    return e.value.code


# ---------------------------------------------------------------- cross attention
def _cross(cache, **change):
    args = dict(scale=1, kv_heads=2, keys=7, K=A, V=2 * A, Q=3 * A, out=4 * A)
    args.update(change)
    return _code(B.amskv_cross_attend, cache, **args)


@pytest.mark.parametrize("native", [True, False], ids=["native", "ctypes"])
def test_cross_attention_refuses_bad_arguments(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_steps", None)
    c = _plan()
    assert _cross(c) == B.ERR_UNSUPPORTED          # all is well, but there is no device memory
    assert _cross(c, keys=1 << 30) == B.ERR_UNSUPPORTED
    assert _cross(None) == B.ERR_INVALID
    for change in (dict(scale=3), dict(scale=-1), dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=8), dict(keys=0), dict(max_keys=-1),
                   dict(K=None), dict(V=None), dict(Q=None), dict(out=None), dict(K=A + 8), dict(Q=A + 2), dict(out=A + 4),
                   dict(lengths=A, offsets=A), dict(lengths=A + 2), dict(offsets=A + 1)):
        assert _cross(c, **change) == B.ERR_INVALID, change
    assert _cross(c, keys=(1 << 30) + 1) == B.ERR_UNSUPPORTED
    kv = torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16)
    assert _cross(c, K=kv[:, :1].expand(2, 2, 7, 64), V=kv[:, :1].expand(2, 2, 7, 64)) == B.ERR_INVALID     # a head repeated
    assert _cross(c, K=kv[:1].expand(2, 2, 7, 64), V=kv[:1].expand(2, 2, 7, 64)) == B.ERR_UNSUPPORTED     # a row repeated is fine
    odd = torch.zeros(2, 2, 7, 68, dtype=torch.bfloat16)[..., :64]
    assert _cross(c, K=odd, V=odd) == B.ERR_INVALID                                                         # strides that are no multiples of 8
    with pytest.raises(ValueError):
        B.amskv_cross_attend(c, 1, 2, 7, kv, odd, 3 * A, 4 * A)
    q = torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16)
    assert _cross(c, out=q[:1].expand(2, 4, 4, 64)) == B.ERR_INVALID
    with pytest.raises(OverflowError):
        B.amskv_cross_attend(c, 1, 2, 1 << 31, A, A, A, A)
    B.amskv_cache_destroy(c)


# ---------------------------------------------------------------- the cache held in 8 bits
@pytest.mark.parametrize("sides", [synth.SIDES_256, synth.SIDES_1024, (4, 8, 1, 3, 12), (1,)])
@pytest.mark.parametrize("policy", [(0, 1, False), (1, 2, False), (2, 3, False), (0, 1, True), (1, 1, B.LAYER_PROMOTABLE)])
def test_segments_start_on_blocks_and_do_not_collide(sides, policy):
    tokens = [s * s for s in sides]
    blocks = [(t + 15) // 16 for t in tokens]
    c, plain = _plan(sides, [policy], flags=B.FLAG_KV_E4M3), _plan(sides, [policy])
    owner, capacity = {}, 0
    for k in range(len(sides)):
        B.amskv_append(c, 0, k, None, None)
        (src, dst, n), = B.amskv_append_copies(c, 0, k)
        assert src == 0 and n == tokens[k] and dst % 16 == 0
        for b in range(blocks[k]):
            owner[dst // 16 + b] = k
        kept = B.amskv_kept_segments(c, 0, k)
        assert kept == B.amskv_kept_segments(plain, 0, k) == oracle.keep_set(k, policy[0], policy[1], policy[2] is True)
        for s in kept:   # no block of a kept segment has a new tenant
            assert sum(v == s for v in owner.values()) == blocks[s]
        ranges = B.amskv_resident_ranges(c, 0, k)
        assert sum(n for _, n in ranges) == sum(tokens[s] for s in kept)
        assert all(a % 16 == 0 for a, _ in ranges) and all(a + n <= b for (a, n), (b, _) in zip(ranges, ranges[1:]))
        assert sum((n + 15) // 16 for _, n in ranges) == sum(blocks[s] for s in kept)
        capacity = max([capacity] + [a + (n + 15) // 16 * 16 for a, n in ranges])
        assert B.amskv_cache_bytes(c)[1] == sum(tokens[s] for s in kept) * 2 * 4 * 64 * 2
    allocated = B.amskv_cache_bytes(c)[0]
    assert allocated >= 256 + capacity * 8 * 2 * 64 + 8 * 2 * capacity // 16
    B.amskv_cache_destroy(c)
    B.amskv_cache_destroy(plain)


def test_half_the_memory():
    d8, _k = B.make_desc(1, 16, 64, 8, synth.SIDES_1024, [(0, 1, True)], flags=B.FLAG_KV_E4M3)
    d16, _k2 = B.make_desc(1, 16, 64, 8, synth.SIDES_1024, [(0, 1, True)])
    assert 0.50 < B.amskv_cache_required_bytes(d8) / B.amskv_cache_required_bytes(d16) < 0.52


def test_what_a_cache_of_8_bits_refuses():
    for flags in (B.FLAG_BULK_APPEND, B.FLAG_TRANSIENT_LAST_SCALE):
        d, _k = B.make_desc(1, 2, 64, 2, (1, 2), [(0, 1, True)], flags=B.FLAG_KV_E4M3 | flags)
        assert _code(B.amskv_cache_create, d) == B.ERR_UNSUPPORTED
    d, _k = B.make_desc(1, 2, 64, 2, (1, 2), [(0, 1, True)], flags=B.FLAG_KV_E4M3, token_budgets=[(5, 1)])
    assert _code(B.amskv_cache_required_bytes, d) == B.ERR_UNSUPPORTED
    d, _k = B.make_desc(1, 2, 64, 2, (1, 2), [(0, 1, True)], flags=16)
    assert _code(B.amskv_cache_required_bytes, d) == B.ERR_INVALID
    d, _k = B.make_desc(1, 2, 64, 2, (1, 2), [(0, 1, True)], flags=B.FLAG_KV_E4M3 | B.FLAG_PLAN_ONLY, token_budgets=[(0, 0)])
    c = B.amskv_cache_create(d)       # a budget of 0 is none
    assert _code(B.amskv_set_attend_path, c, B.PATH_SIMT) == B.ERR_UNSUPPORTED
    B.amskv_set_attend_path(c, B.PATH_SMALL)
    B.amskv_append(c, 0, 0, None, None)
    assert _code(B.amskv_attention_density, c, 0, 0, A, A, 100) == B.ERR_UNSUPPORTED
    assert _code(B.amskv_attend_density, c, 0, 0, A, 2 * A, 3 * A, 100) == B.ERR_UNSUPPORTED
    B.amskv_cache_destroy(c)


@pytest.mark.parametrize("flags", [0, B.FLAG_KV_E4M3])
def test_reading_a_segment_refuses_what_is_not_there(flags):
    c = _plan((1, 2, 3, 4), [(1, 1, False)], flags=flags)
    assert _code(B.amskv_read_segment, c, 0, 0, A, 2 * A) == B.ERR_ORDER
    for k in range(3):
        B.amskv_append(c, 0, k, None, None)
    assert B.amskv_kept_segments(c, 0, 2) == [0, 2]
    assert _code(B.amskv_read_segment, c, 0, 1, A, 2 * A) == B.ERR_ORDER       # evicted
    assert _code(B.amskv_read_segment, c, 0, 3, A, 2 * A) == B.ERR_ORDER       # not there yet
    assert _code(B.amskv_read_segment, c, 0, 2, A, 2 * A) == B.ERR_UNSUPPORTED  # plan only
    for bad in ((1, 0, A, A), (0, 4, A, A), (0, -1, A, A), (0, 2, None, A), (0, 2, A, A + 8)):
        assert _code(B.amskv_read_segment, c, *bad) == B.ERR_INVALID, bad
    x = torch.zeros(1, 4, 9, 64, dtype=torch.bfloat16).expand(2, 4, 9, 64)
    assert _code(B.amskv_read_segment, c, 0, 2, x, x) == B.ERR_INVALID
    B.amskv_cache_destroy(c)
    c = _plan((1, 2), [(1, 1, False)], token_budgets=[(5, 1)])
    B.amskv_append(c, 0, 0, None, None)
    assert _code(B.amskv_read_segment, c, 0, 0, A, 2 * A) == B.ERR_UNSUPPORTED
    B.amskv_cache_destroy(c)


def test_promotion_of_a_layer_held_in_8_bits():
    c = _plan((1, 2, 3, 4), [(1, 1, B.LAYER_PROMOTABLE)], flags=B.FLAG_KV_E4M3)
    B.amskv_append(c, 0, 0, None, None)
    B.amskv_append(c, 0, 1, None, None)
    before = B.amskv_resident_ranges(c, 0, 1)
    B.amskv_promote_layer(c, 0)
    assert B.amskv_resident_ranges(c, 0, 1) == before     # nothing moves
    B.amskv_append(c, 0, 2, None, None)
    assert B.amskv_kept_segments(c, 0, 2) == [0, 1, 2]
    assert B.amskv_resident_ranges(c, 0, 2) == [(0, 1), (16, 4), (32, 9)]
    assert np.isfinite(B.amskv_cache_bytes(c)).all()
    B.amskv_cache_destroy(c)


@pytest.mark.parametrize("native", [True, False], ids=["native", "ctypes"])
def test_lengths_and_offsets_that_the_kernels_would_misread(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_steps", None)
    c = _plan()                                   # two rows
    q = torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    for kw in (dict(lengths=torch.zeros(2, **i32)), dict(lengths=torch.zeros(5, **i32)), dict(offsets=torch.zeros(3, **i32)), dict(lengths=A),
               dict(offsets=torch.zeros(1, **i32), Q=3 * A), dict(lengths=None)):
        assert _cross(c, **{**dict(Q=q), **kw}) == B.ERR_UNSUPPORTED, kw     # all is well, but there is no device memory
    for kw in (dict(lengths=torch.zeros(2, dtype=torch.int64)), dict(lengths=torch.cumsum(torch.ones(2, **i32), 0)), dict(lengths=torch.zeros(2)),
               dict(offsets=torch.zeros(3, dtype=torch.int64)), dict(lengths=torch.zeros(1, **i32)), dict(lengths=torch.zeros(0, **i32)),
               dict(offsets=torch.zeros(2, **i32)), dict(lengths=torch.zeros(2, dtype=torch.int16))):
        for queries in (q, q.transpose(1, 2).contiguous().transpose(1, 2)):
            with pytest.raises(ValueError):
                B.amskv_cross_attend(c, 1, 2, 7, A, 2 * A, queries, 4 * A, **kw)
    with pytest.raises(ValueError):
        B.amskv_cross_attend(c, 1, 2, 7, A, 2 * A, 3 * A, 4 * A, lengths=torch.zeros(2, dtype=torch.int64))
    B.amskv_cache_destroy(c)


def test_the_row_stride_of_packed_keys_is_not_looked_at():
    c = _plan()
    kv = torch.zeros(4096, dtype=torch.bfloat16)
    for row in (3, 0, 1 << 20):
        x = torch.as_strided(kv, (1, 2, 7, 64), (row, 64, 128, 1))
        assert _cross(c, K=x, V=x, offsets=A) == B.ERR_UNSUPPORTED       # all is well, but there is no device memory
    strides = (B.ctypes.c_int64 * 3)(-8, 64, 128)
    enc = B.Encoder(2, 7, 0, None, A)
    assert B.lib.amskv_cross_attend(c, 1, B.ctypes.byref(enc), A, A, strides, A, 2 * A, None, None, None) == B.ERR_UNSUPPORTED
    x = torch.as_strided(kv, (1, 2, 7, 64), (3, 64, 128, 1))
    assert _cross(c, K=x, V=x) == B.ERR_INVALID                          # padded keys: it is
    x = torch.as_strided(kv, (1, 2, 7, 64), (0, 0, 128, 1))
    assert _cross(c, K=x, V=x, offsets=A) == B.ERR_INVALID               # a head repeated
    B.amskv_cache_destroy(c)
