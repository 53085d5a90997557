"""Cross attention to an encoder's states on the GPU against the definition in 64 bits.

Tolerance, element by element: half a step of bf16 of the output (2^-8), and the probabilities' rounding to bf16, 2^-8 of the sum
of p |v|, and the exponentials' own error, 2^-10 at most (a cubic in one kernel; the special-function unit's is 2^-22), of the same
sum in numerator and denominator."""
import math

import numpy as np
import pytest
import torch

from gpu_common import Cache
from oracle import operators as ref
from paper_2511_16047_b200 import binding as B

pytestmark = pytest.mark.gpu

PATHS = {"auto": B.PATH_AUTO, "rows": B.PATH_SMALL, "tiles": B.PATH_TENSOR_PAIR}


def _np(x):
    return x.detach().cpu().double().numpy()


def _check(out, q, keys, group, scale, what):
    """keys[r] = (k, v) of row r: [kv_heads, n, D] in 64 bits."""
    got = _np(out)
    for r, (k, v) in enumerate(keys):
        k, v = np.repeat(k, group, 0), np.repeat(v, group, 0)
        want, size = ref.attention(_np(q[r]), k, v, scale)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -9) * size
        assert (np.abs(got[r] - want) <= tol).all(), (what, r, np.abs(got[r] - want).max(), (np.abs(got[r] - want) / (tol + 1e-30)).max())


def _lengths(rows, keys):
    """None, one, a few, one short of a block, of a tile, all."""
    pool = [keys, 0, 1, min(15, keys), min(17, keys), min(63, keys), min(65, keys), (keys + 1) // 2, max(keys - 1, 0)]
    return [pool[r % len(pool)] for r in range(rows)]


SHAPES = [
    # rows, heads, kv_heads, D, side, keys
    (1, 1, 1, 64, 1, 1),
    (2, 16, 16, 128, 1, 77),
    (9, 4, 2, 64, 1, 200),
    (9, 8, 2, 128, 2, 130),        # a group of heads fills one block of query rows
    (3, 6, 2, 64, 3, 64),          # 27 rows of a group: two blocks
    (9, 3, 3, 64, 5, 77),
    (9, 4, 4, 128, 6, 512),
    (2, 5, 1, 64, 7, 40),
    (4, 3, 3, 64, 11, 129),        # 121 queries: one tile
    (4, 3, 3, 128, 11, 300),
    (5, 5, 5, 64, 13, 81),         # 169 queries: two tiles, an odd number of heads
    (5, 3, 1, 128, 13, 190),
    (9, 3, 3, 64, 18, 333),        # 324 queries: three tiles
    (3, 3, 3, 128, 20, 65),
    (2, 2, 2, 128, 32, 1100),
    # CTAs of two and of four 16-row blocks
    (10, 4, 4, 64, 11, 200),
    (8, 5, 5, 128, 11, 600),
    (100, 3, 3, 64, 5, 150),
    (100, 3, 3, 128, 9, 90),
    # several units per CTA: streams with tiles of their own, and (an odd number of them) one alone in a unit
    (40, 16, 16, 128, 2, 150),
    (110, 3, 3, 128, 2, 130),
    (130, 5, 5, 64, 2, 100),
    (50, 3, 1, 128, 16, 70),
]


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_rows_of_different_lengths(shape, path):
    rows, heads, kv, D, side, keys = shape
    T, group = side * side, heads // kv
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    q = torch.randn(rows, heads, T, D, generator=g, device="cuda").bfloat16()
    lengths = _lengths(rows, keys)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(rows, kv, keys, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    behind = torch.arange(keys, device="cuda")[None] >= n[:, None]
    k[behind[:, None].expand(rows, kv, keys)] = float("nan")       # what lies behind a row's last key is never looked at
    v[behind[:, None].expand(rows, kv, keys)] = float("inf")
    want = [(_np(k[r, :, :m]), _np(v[r, :, :m])) for r, m in enumerate(lengths)]
    scale = 1.0 / math.sqrt(D)
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        out = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, kv, keys, k, v, q, out, lengths=n)
        assert B.amskv_status(c.h) == 0
        _check(out, q, want, group, scale, "padded")
        again = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, kv, keys, k, v, q, again, lengths=n)
        assert torch.equal(out, again)

        # packed, all tensors views of what projections leave, and guard values around the output
        total = sum(lengths)
        kv2 = torch.full((total + 3, 2, kv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        at = 0
        for r, m in enumerate(lengths):
            kv2[at:at + m, 0], kv2[at:at + m, 1] = k[r, :, :m].transpose(0, 1), v[r, :, :m].transpose(0, 1)
            at += m
        off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
        kp, vp = (kv2[:, i].transpose(0, 1)[None] for i in range(2))
        qv = q.transpose(1, 2).contiguous().transpose(1, 2)
        big = torch.full((rows, T + 1, heads + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
        ov = big[:, :T, 1:].transpose(1, 2)
        B.amskv_cross_attend(c.h, 0, kv, total + 3, kp, vp, qv, ov, offsets=off, max_keys=max(lengths))
        assert B.amskv_status(c.h) == 0
        _check(ov, q, want, group, scale, "packed")
        assert (big[:, T] == 7.0).all() and (big[:, :, 0] == 7.0).all()


@pytest.mark.parametrize("path", sorted(PATHS))
def test_all_keys_the_same_keys_for_all_rows_and_cut_lengths(path):
    rows, heads, kv, D, side, keys = 3, 4, 2, 64, 12, 100
    q = torch.randn(rows, heads, side * side, D, device="cuda").bfloat16()
    k, v = (torch.randn(1, kv, keys, D, device="cuda").bfloat16() for _ in range(2))
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)], softmax_scale=0.3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])

        def run(**kw):
            out = torch.full_like(q, float("nan"))
            B.amskv_cross_attend(c.h, 0, kv, keys, kk, vv, q, out, **kw)
            assert B.amskv_status(c.h) == 0
            return out

        def want(counts, firsts=(0, 0, 0)):
            return [(_np(kk[r % kk.shape[0], :, f:f + n]), _np(vv[r % kk.shape[0], :, f:f + n])) for r, (n, f) in enumerate(zip(counts, firsts))]

        kk, vv = k.expand(rows, kv, keys, D), v.expand(rows, kv, keys, D)
        _check(run(), q, want([100] * 3), 2, 0.3, "broadcast")
        kk, vv = kk.contiguous(), vv.contiguous()
        _check(run(), q, want([100] * 3), 2, 0.3, "all keys")
        _check(run(max_keys=70), q, want([70] * 3), 2, 0.3, "cut to max_keys")
        odd = torch.tensor([-5, 1 << 30, 33], dtype=torch.int32, device="cuda")     # lengths outside the tensor are cut to it
        _check(run(lengths=odd), q, want([0, 100, 33]), 2, 0.3, "odd lengths")
        kk, vv = k, v
        off = torch.tensor([-7, 20, 12, 1 << 30], dtype=torch.int32, device="cuda")  # from 0 to 20, none, from 12 to the end
        _check(run(offsets=off), q, want([20, 0, 88], [0, 0, 12]), 2, 0.3, "odd offsets")
        off = torch.tensor([2 ** 31 - 1, -2 ** 31, 100, 100], dtype=torch.int32, device="cuda")
        _check(run(offsets=off), q, want([0, 100, 0], [0, 0, 0]), 2, 0.3, "offsets in no order")


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
def test_peaked_logits_and_large_values(path, D):
    """Logits tens apart, growing from tile to tile so that the reference has to move, and values of very different sizes."""
    rows, heads, side, keys = 2, 2, 14, 400
    g = torch.Generator(device="cuda").manual_seed(D)
    q = (6.0 * torch.randn(rows, heads, side * side, D, generator=g, device="cuda")).bfloat16()
    k = torch.randn(rows, heads, keys, D, generator=g, device="cuda")
    k = (k * (torch.arange(keys, device="cuda")[:, None] / 100.0)).bfloat16()
    v = (torch.randn(rows, heads, keys, D, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (1, 1, keys, 1), generator=g, device="cuda").float())).bfloat16()
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        out = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, out)
        assert B.amskv_status(c.h) == 0
        _check(out, q, [(_np(k[r]), _np(v[r])) for r in range(rows)], 1, 1.0 / math.sqrt(D), "peaked")


def test_the_cache_is_left_alone_and_order_does_not_matter():
    """Cross attention between the steps of a layer, on another stream, and captured: the cache's own results stay the same."""
    sides, heads, D, rows, keys = (1, 2, 4), 2, 64, 2, 33
    steps = [[torch.randn(rows, heads, s * s, D, device="cuda").bfloat16() for _ in range(3)] for s in sides]
    k, v = (torch.randn(rows, heads, keys, D, device="cuda").bfloat16() for _ in range(2))
    with Cache(1, heads, D, rows, sides, [(0, 1, True)]) as c:
        outs = []
        for cross in (False, True):
            B.amskv_cache_reset(c.h)
            outs.append([])
            for i, (q, kk, vv) in enumerate(steps):
                o = torch.empty_like(q)
                B.amskv_append_attend(c.h, 0, i, kk, vv, q, o)
                outs[-1].append(o)
                if cross:
                    for s in range(len(sides)):
                        x = torch.full_like(steps[s][0], float("nan"))
                        B.amskv_cross_attend(c.h, s, heads, keys, k, v, steps[s][0], x)
                        _check(x, steps[s][0], [(_np(k[r]), _np(v[r])) for r in range(rows)], 1, 0.125, "between steps")
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        q = steps[2][0]
        x = torch.empty_like(q)
        B.amskv_cross_attend(c.h, 2, heads, keys, k, v, q, x, stream=side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.amskv_cross_attend(c.h, 2, heads, keys, k, v, q, x, stream=side)
        q.copy_(torch.randn_like(q))
        k.copy_(torch.randn_like(k))
        x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        _check(x, q, [(_np(k[r]), _np(v[r])) for r in range(rows)], 1, 0.125, "replayed")
        assert B.amskv_status(c.h) == 0


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("side", [2, 12])
def test_offsets_beyond_32_bits(side, path):
    """Rows of queries, outputs, keys and values 2^31 + 64 values apart."""
    rows, heads, D, keys, apart = 3, 2, 64, 70, (1 << 31) + 64
    T = side * side
    base = torch.empty(2 * apart + 8 * heads * (keys + T) * D, dtype=torch.bfloat16, device="cuda")
    one, two = heads * keys * D, heads * T * D
    k, v = (torch.as_strided(base, (rows, heads, keys, D), (apart, keys * D, D, 1), n * one) for n in range(2))
    q, o = (torch.as_strided(base, (rows, heads, T, D), (apart, T * D, D, 1), 2 * one + n * two) for n in range(2))
    for x in (k, v, q):
        x.copy_(torch.randn(x.shape, device="cuda"))
    o.fill_(float("nan"))
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, o)
        _check(o, q, [(_np(k[r]), _np(v[r])) for r in range(rows)], 1, 0.125, "far")
        assert B.amskv_status(c.h) == 0


def test_one_cache_on_two_streams():
    """Cross attention reads nothing of the cache but its shapes, so that calls of one cache may overlap."""
    rows, heads, D, keys, side = 4, 20, 128, 300, 12
    streams = [torch.cuda.Stream() for _ in range(2)]
    q, k, v = ([torch.randn(rows, heads, n, D, device="cuda").bfloat16() for _ in range(2)] for n in (side * side, keys, keys))
    outs = [[torch.empty_like(x) for x in q] for _ in range(4)]
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        torch.cuda.synchronize()
        for j in range(2):
            B.amskv_cross_attend(c.h, 0, heads, keys, k[j], v[j], q[j], outs[0][j])
        torch.cuda.synchronize()
        for out in outs[1:]:
            for j in range(2):
                B.amskv_cross_attend(c.h, 0, heads, keys, k[j], v[j], q[j], out[j], stream=streams[j])
        torch.cuda.synchronize()
        assert B.amskv_status(c.h) == 0
    for out in outs[1:]:
        assert torch.equal(out[0], outs[0][0]) and torch.equal(out[1], outs[0][1])


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("growth", [0.0, 15.0, 40.0])
@pytest.mark.parametrize("power", [100, -60])
def test_large_and_small_values_behind_a_maximum_that_grows(power, growth, path, D):
    """Logits near 0 in the first 64 keys and near `growth` behind: sums against the first keys' maximum have to stay in fp32 with
    values near 2^100, and to be kept with values near 2^-60."""
    rows, heads, side, keys = 2, 2, 12, 200
    g = torch.Generator(device="cuda").manual_seed(D)
    q = 0.1 * torch.randn(rows, heads, side * side, D, generator=g, device="cuda")
    k, v = (torch.randn(rows, heads, keys, D, generator=g, device="cuda") for _ in range(2))
    q[..., 0], k[..., 0], k[:, :, 64:, 0] = 1.0, 0.0, growth * math.sqrt(D)
    q, k, v = (x.bfloat16() for x in (q, k, v * 2.0 ** power))
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        out = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, out)
        assert B.amskv_status(c.h) == 0
        _check(out, q, [(_np(k[r]), _np(v[r])) for r in range(rows)], 1, 1.0 / math.sqrt(D), "outgrown")


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
def test_a_number_that_is_none_is_not_lost(path, D):
    """A NaN in a key makes every output of its (row, head) one, a NaN in a value that channel's, wherever the key lies in its tile;
    no other output changes."""
    rows, heads, kv, side, keys = 2, 4, 2, 12, 200
    g = torch.Generator(device="cuda").manual_seed(D)
    q = torch.randn(rows, heads, side * side, D, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(rows, kv, keys, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    n = torch.tensor([keys, 150], dtype=torch.int32, device="cuda")
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])

        def run(kk, vv):
            out = torch.zeros_like(q)
            B.amskv_cross_attend(c.h, 0, kv, keys, kk, vv, q, out, lengths=n)
            assert B.amskv_status(c.h) == 0
            return out

        plain = run(k, v)
        assert torch.isfinite(plain).all()
        for at in [*range(0, 28), 36, 48, 60, 63, 64, 76, 128, 149]:
            kk, vv = k.clone(), v.clone()
            kk[1, 0, at, 3] = float("nan")
            out = run(kk, v)
            assert torch.isnan(out[1, :2]).all(), at
            assert torch.equal(out[0], plain[0]) and torch.equal(out[1, 2:], plain[1, 2:]), at
            vv[0, 1, at, 7] = float("nan")
            out = run(k, vv)
            assert torch.isnan(out[0, 2:, :, 7]).all(), at
            out[0, 2:, :, 7] = plain[0, 2:, :, 7]
            assert torch.equal(out, plain), at


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D,kv,side,keys", [(64, 4, 1, 600), (64, 2, 3, 1100), (64, 4, 10, 130), (128, 4, 4, 600), (128, 1, 12, 200)])
def test_a_path_of_ones_own_choice_depends_on_the_shapes_alone(D, kv, side, keys, path):
    """Under every path but AUTO an image has the same outputs whatever other images it is computed with, bit for bit."""
    heads, most = 4, 90
    g = torch.Generator(device="cuda").manual_seed(D + keys)
    q = torch.randn(most, heads, side * side, D, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(most, kv, keys, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    n = torch.tensor(_lengths(most, keys), dtype=torch.int32, device="cuda")
    want = None
    for rows in (most, 1, 2, 9, 30):
        with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
            B.amskv_set_attend_path(c.h, PATHS[path])
            out = torch.zeros_like(q[:rows])
            B.amskv_cross_attend(c.h, 0, kv, keys, k[:rows], v[:rows], q[:rows], out, lengths=n[:rows])
            assert B.amskv_status(c.h) == 0
        want = out if want is None else want
        assert torch.equal(out, want[:rows]), rows


@pytest.mark.parametrize("shape", [(3, 1, 1, 64, 20, 512), (2, 4, 2, 64, 2, 700), (2, 4, 2, 64, 2, 1300), (3, 2, 2, 64, 15, 520),
                                   (2, 4, 2, 128, 2, 700), (2, 4, 2, 128, 2, 1300), (3, 2, 1, 128, 7, 520)], ids=lambda s: "x".join(map(str, s)))
def test_clusters_that_share_long_keys(shape):
    """Two, four and eight CTAs to a row's keys, which only calls of few items under AUTO have."""
    test_rows_of_different_lengths(shape, "auto")


@pytest.mark.parametrize("D,group,side,rows,tiles", [
    (64, 8, 2, 80, False), (64, 2, 4, 200, False), (64, 4, 3, 40, False), (64, 8, 5, 80, False), (64, 4, 6, 200, True), (64, 1, 6, 200, True),
    (128, 8, 2, 80, False), (128, 2, 4, 80, False), (128, 8, 4, 200, False), (128, 4, 5, 80, True), (128, 4, 10, 80, True)])
def test_few_queries_of_grouped_heads_share_a_block(D, group, side, rows, tiles):
    """Which kernel AUTO takes, told by the bits of its outputs: a tile of 128 rows holds one head's queries, a block of the
    warp-matrix kernel those of all heads that share a key."""
    kv, keys = 8, 200
    g = torch.Generator(device="cuda").manual_seed(group)
    q = torch.randn(rows, kv * group, side * side, D, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(rows, kv, keys, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    outs = []
    with Cache(1, kv * group, D, rows, (side,), [(0, 1, False)]) as c:
        for path in (B.PATH_AUTO, B.PATH_TENSOR_PAIR):
            B.amskv_set_attend_path(c.h, path)
            outs.append(torch.zeros_like(q))
            B.amskv_cross_attend(c.h, 0, kv, keys, k, v, q, outs[-1])
        assert B.amskv_status(c.h) == 0
    assert torch.equal(*outs) == tiles
    at = [0, rows - 1]
    _check(outs[0][at], q[at], [(_np(k[r]), _np(v[r])) for r in at], group, 1.0 / math.sqrt(D), "grouped")


@pytest.mark.parametrize("D,heads,side,rows", [(64, 8, 8, 100), (64, 8, 6, 100), (128, 4, 13, 3), (128, 4, 16, 2), (64, 4, 1, 2)])
def test_what_the_cache_holds_makes_no_difference(D, heads, side, rows):
    """Cross attention takes the kernel that an encoder's keys are best served by, beside a cache of 8 bits as beside any other."""
    keys = 200
    g = torch.Generator(device="cuda").manual_seed(side)
    q = torch.randn(rows, heads, side * side, D, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(rows, heads, keys, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    outs = []
    for flags in (0, B.FLAG_KV_E4M3):
        with Cache(1, heads, D, rows, (side,), [(0, 1, False)], flags=flags) as c:
            outs.append(torch.zeros_like(q))
            B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, outs[-1])
            assert B.amskv_status(c.h) == 0
    assert torch.equal(*outs)


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("after", [0.0, -500.0, 30.0])
@pytest.mark.parametrize("masked", [1, 63, 64, 130])
def test_scores_of_minus_infinity(masked, after, path, D):
    """Keys masked by an infinity in one channel: tiles of nothing else first, logits of any size behind them, and masked keys among those."""
    rows, heads, side, keys = 2, 2, 12, 200
    g = torch.Generator(device="cuda").manual_seed(masked)
    q = torch.randn(rows, heads, side * side, D, generator=g, device="cuda")
    k, v = (torch.randn(rows, heads, keys, D, generator=g, device="cuda") for _ in range(2))
    q[..., 0], q[..., 1], k[..., 0], k[..., 1] = 1.0, 1.0, 0.0, after * math.sqrt(D)
    real = torch.ones(keys, dtype=torch.bool)
    real[:masked] = real[150:160] = False
    k[:, :, ~real, 0] = -float("inf")
    q, k, v = (x.bfloat16() for x in (q, k, v))
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)]) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        out = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, out)
        assert B.amskv_status(c.h) == 0
        _check(out, q, [(_np(k[r][:, real]), _np(v[r][:, real])) for r in range(rows)], 1, 1.0 / math.sqrt(D), "masked")
        k[..., 0] = -float("inf")                            # of all keys: none is left, and the row gets zeros
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, out)
        assert B.amskv_status(c.h) == 0 and (out == 0).all()


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [0.3, 1.0, 4.0])
def test_errors_in_the_mean_are_those_of_two_roundings(spread, D, path):
    """Root mean square over all outputs.  A bf16 rounding is off by up to 2^-8 / m of a number m 2^e, evenly: in the mean over mantissas
    spread as those of products are, 2^-8 * 0.735 / sqrt(3) = 0.85 * 2^-9 of it.  The output is rounded once, and each probability once
    before it meets its value.  The cubic adds 2^-10 of one pair in six at most, 0.03 of that in squares."""
    rows, heads, side, keys = 2, 4, 16, 500
    g = torch.Generator(device="cuda").manual_seed(D)
    q, k, v = (torch.randn(rows, heads, n, D, generator=g, device="cuda").bfloat16() for n in (side * side, keys, keys))
    scale = spread / math.sqrt(D)
    with Cache(1, heads, D, rows, (side,), [(0, 1, False)], softmax_scale=scale) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        out = torch.full_like(q, float("nan"))
        B.amskv_cross_attend(c.h, 0, heads, keys, k, v, q, out)
        assert B.amskv_status(c.h) == 0
    p = torch.softmax(scale * (q.double() @ k.double().transpose(2, 3)), -1)
    want, spread_of_p = p @ v.double(), (p * p) @ (v.double() * v.double())
    rms = float((out.double() - want).square().mean().sqrt())
    assert rms <= 2.0 ** -9 * float((want.square() + spread_of_p).mean().sqrt()), rms
