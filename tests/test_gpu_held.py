"""A cache held in 8 bits on the GPU against the definition in 64 bits: what it holds, bit for bit, and attention over it.

Tolerance of the attention, element by element: as for cross attention -- half a step of bf16 of the output, 2^-8 of the sum of
p |v| for the probabilities' rounding, 2^-9 of it for the exponentials' own."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_common import Cache
from oracle import operators as ref
from paper_2511_16047_b200 import binding as B
from paper_2511_16047_b200 import synth

pytestmark = pytest.mark.gpu

PATHS = {"auto": B.PATH_AUTO, "rows": B.PATH_SMALL, "tiles": B.PATH_TENSOR_PAIR}


def _np(x):
    return x.detach().cpu().double().numpy()


def _steps(rows, heads, sides, D, seed):
    """Keys with large channels, heads of very different sizes, a head of zeros now and then, tiny values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, s in enumerate(sides):
        q, k, v = (torch.randn(rows, heads, s * s, D, generator=g, device="cuda") for _ in range(3))
        k[..., ::9] *= 5.0
        v *= torch.exp2(torch.randint(-12, 12, (rows, heads, 1, 1), generator=g, device="cuda").float())
        v[..., ::5] *= 2.0 ** -9           # codes below the least with a leading one
        if i % 3 == 1:
            v[-1, -1] = 0.0
        out.append([x.bfloat16() for x in (q, k, v)])
    return out


def _views(x):
    r, h, t, d = x.shape
    y = torch.full((r, t, 3, h, d), 7.0, dtype=x.dtype, device=x.device)
    y[:, :, 1] = x.transpose(1, 2)
    return y[:, :, 1].transpose(1, 2)


def _check(out, q, ks, vs, kept, scale, what):
    k, v = np.concatenate([ks[s] for s in kept], -2), np.concatenate([vs[s] for s in kept], -2)
    want, size = ref.attention(_np(q), k, v, scale)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -9) * size
    err = np.abs(_np(out) - want)
    assert (err <= tol).all(), (what, err.max(), (err / (tol + 1e-300)).max())


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("rows,heads,D,sides,policy", [
    (1, 1, 64, (1,), (0, 1, False)),
    (2, 3, 64, synth.SIDES_256, (2, 2, False)),
    (2, 2, 128, synth.SIDES_256, (1, 3, False)),
    (1, 3, 64, (1, 3, 5, 7, 9, 11, 15, 19), (0, 1, True)),
    (3, 1, 128, (4, 8, 12, 13, 18), (0, 1, True)),
    (1, 2, 64, (9, 2, 14, 1, 3), (1, 1, False)),       # scales that shrink: few queries, many keys
    (1, 2, 128, (20, 1, 4), (0, 1, True)),
    (110, 3, 128, (2, 7, 3), (0, 1, True)),            # several units per CTA, a stream alone in every other one
    (80, 9, 64, (3, 5), (0, 1, True)),
    (4, 10, 64, (3, 12, 13), (0, 1, True)),            # an SM for each CTA of 64 query rows, with and without a share of the keys
    (4, 5, 128, (3, 12, 13), (0, 1, True)),
    (10, 12, 128, (3, 6, 8), (0, 1, True)),
])
def test_a_schedule(rows, heads, D, sides, policy, path):
    steps = _steps(rows, heads, sides, D, sum(sides) + D)
    scale = 1.0 / math.sqrt(D)
    ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
    with Cache(1, heads, D, rows, sides, [policy], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        for views in (False, True):
            B.amskv_cache_reset(c.h)
            for i, (q, k, v) in enumerate(steps):
                kept = oracle.keep_set(i, *policy)
                if views:
                    kk, vv, qq, o = _views(k), _views(v), _views(q), _views(torch.zeros_like(q))
                    B.amskv_append_attend(c.h, 0, i, kk, vv, qq, o)
                    assert (o._base[:, :, 0] == 7.0).all() and (o._base[:, :, 2] == 7.0).all()
                else:
                    o = torch.full_like(q, float("nan"))
                    B.amskv_append(c.h, 0, i, k, v)
                    B.amskv_attend(c.h, 0, i, q, o)
                assert B.amskv_status(c.h) == 0
                _check(o, q, ks, vs, kept, scale, (views, i))
                if not views:
                    again = torch.full_like(q, float("nan"))
                    B.amskv_attend(c.h, 0, i, q, again)
                    assert torch.equal(o, again)
                for s in kept:      # every retained segment comes back as it went in, by block
                    kb, vb = (torch.full((rows, heads, sides[s] ** 2, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
                    if views:
                        kb, vb = _views(kb), _views(vb)
                    B.amskv_read_segment(c.h, 0, s, kb, vb)
                    assert (_np(kb) == ks[s]).all() and (_np(vb) == vs[s]).all(), (i, s)
                    if views:
                        assert (kb._base[:, :, 0] == 7.0).all() and (vb._base[:, :, 2] == 7.0).all()


def test_every_code_and_every_power():
    """Values on and between codes at the ends of the range of powers, ties among them."""
    D, T = 64, 16
    half = torch.arange(0, 128, device="cuda").to(torch.uint8).view(torch.float8_e4m3fn).float()
    codes = half[:127]                                                       # 0 .. 448
    mids = (codes[1:] + codes[:-1]) / 2
    x = torch.cat([codes, -codes, mids, -mids, torch.full((1024 - 506,), 448.0, device="cuda")]).view(1, 1, T, D)
    powers = [-100, -60, -7, -1, 0, 1, 5, 30, 100, 117]
    big = torch.cat([x * 2.0 ** p for p in powers], 0).bfloat16()             # a row for every power
    tiny = torch.full((1, 1, T, D), 2.0 ** -112, device="cuda").bfloat16()    # below half the least code of the least power
    k = torch.cat([big, tiny, torch.zeros_like(tiny)], 0)
    rows = k.shape[0]
    with Cache(1, 1, D, rows, (4,), [(0, 1, False)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_append(c.h, 0, 0, k, -k)
        kb, vb = torch.empty_like(k), torch.empty_like(k)
        B.amskv_read_segment(c.h, 0, 0, kb, vb)
        want = ref.held_values(_np(k))
        assert (_np(kb) == want).all() and (_np(vb) == -want).all()
        assert (want[-2:] == 0).all() and np.abs(want[:-2]).max((1, 2, 3)).tolist() == [448.0 * 2.0 ** p for p in powers]


def test_reading_a_bf16_cache_back():
    sides, rows, heads, D = (1, 3, 5, 2), 2, 3, 128
    steps = _steps(rows, heads, sides, D, 5)
    with Cache(2, heads, D, rows, sides, [(1, 2, False), (0, 1, True)]) as c:
        for i, (q, k, v) in enumerate(steps):
            for layer in range(2):
                B.amskv_append(c.h, layer, i, k, v)
                for s in B.amskv_kept_segments(c.h, layer, i):
                    kb, vb = _views(torch.zeros_like(steps[s][1])), _views(torch.zeros_like(steps[s][1]))
                    B.amskv_read_segment(c.h, layer, s, kb, vb)
                    assert torch.equal(kb, steps[s][1]) and torch.equal(vb, steps[s][2])


def test_layers_rows_and_streams_keep_apart():
    """Two layers of different policies in one graph, another set of inputs on replay, and a host step."""
    sides, rows, heads, D = (1, 2, 3, 6), 2, 2, 64
    pols = [(1, 1, False), (0, 1, True)]
    with Cache(2, heads, D, rows, sides, pols, flags=B.FLAG_KV_E4M3) as c:
        steps = _steps(rows, heads, sides, D, 1)
        outs = [[torch.zeros_like(q) for q, _, _ in steps] for _ in pols]
        side = torch.cuda.Stream()

        def calls():
            B.amskv_cache_reset(c.h)
            for i, (q, k, v) in enumerate(steps):
                for layer in range(2):
                    B.amskv_append_attend(c.h, layer, i, k, v, q, outs[layer][i], side)

        side.wait_stream(torch.cuda.current_stream())
        calls()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
        new = _steps(rows, heads, sides, D, 2)
        for old, fresh in zip(steps, new):
            for a, b in zip(old, fresh):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
        for layer, pol in enumerate(pols):
            for i, (q, _, _) in enumerate(steps):
                _check(outs[layer][i], q, ks, vs, oracle.keep_set(i, *pol), 0.125, (layer, i))
        B.amskv_cache_reset(c.h)
        n = B.amskv_step_staging_bytes(c.h)
        staging = torch.empty(n, dtype=torch.uint8, device="cuda")
        q, k, v = (x.cpu().pin_memory() for x in steps[0])
        o = torch.empty_like(q).pin_memory()
        B.amskv_step_host(c.h, 0, 0, k, v, q, o, staging, n)
        torch.cuda.synchronize()
        _check(o, steps[0][0], ks, vs, [0], 0.125, "host")
        assert B.amskv_status(c.h) == 0


@pytest.mark.parametrize("path", sorted(PATHS))
def test_a_layer_as_it_is_used(path):
    """Rotary positions, the cache of 8 bits, cross attention: one layer of a text-conditioned next-scale transformer."""
    sides, rows, heads, D, keys = (1, 2, 4, 7, 12), 2, 4, 64, 50
    steps = _steps(rows, heads, sides, D, 11)
    tokens = [s * s for s in sides]
    pos = torch.cat([torch.stack(torch.meshgrid(*[torch.arange(s, device="cuda") * (12.0 / s)] * 2, indexing="ij"), -1).reshape(-1, 2) for s in sides])
    spec = B.make_rotary(D, axes=2)
    table = torch.empty(len(pos), D // 2, 2, device="cuda")
    B.amskv_rotary_table(spec, pos.float().contiguous(), len(pos), table)
    ek, ev = (torch.randn(rows, heads, keys, D, device="cuda").bfloat16() for _ in range(2))
    n = torch.tensor([keys, 3], dtype=torch.int32, device="cuda")
    angles = ref.rotary_angles(pos.cpu().numpy(), D)
    ks, vs = [], []
    with Cache(1, heads, D, rows, sides, [(1, 2, False)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        first = 0
        for i, (q, k, v) in enumerate(steps):
            T = tokens[i]
            qr, kr = torch.empty_like(q), torch.empty_like(k)
            B.amskv_rotary(spec, table, len(pos), first, None, rows, T, D, heads, q, qr, heads, k, kr)
            want = ref.rotate(_np(k), angles[first:first + T], 2)
            assert (np.abs(_np(kr) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * 64).all()
            out, cross = torch.empty_like(q), torch.empty_like(q)
            B.amskv_append_attend(c.h, 0, i, kr, v, qr, out)
            B.amskv_cross_attend(c.h, i, heads, keys, ek, ev, out, cross, lengths=n)
            assert B.amskv_status(c.h) == 0
            ks.append(ref.held_values(_np(kr)))
            vs.append(ref.held_values(_np(v)))
            _check(out, qr, ks, vs, oracle.keep_set(i, 1, 2, False), 0.125, i)
            for r, m in enumerate((keys, 3)):
                w, size = ref.attention(_np(out[r]), _np(ek[r, :, :m]), _np(ev[r, :, :m]), 0.125)
                assert (np.abs(_np(cross[r]) - w) <= 2.0 ** -8 * np.abs(w) + (2.0 ** -8 + 2.0 ** -9) * size).all()
            first += T


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_more_keys_than_the_tables_of_a_launch(D, path):
    """12 544 keys, and more behind them with a short block between: tiles beyond the 192 that a launch tabulates."""
    sides, rows, heads = (112, 3, 12, 2), 1, 3
    steps = _steps(rows, heads, sides, D, D)
    ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        B.amskv_append(c.h, 0, 0, steps[0][1], steps[0][2])
        for i in (1, 2, 3):
            q, k, v = steps[i]
            o = torch.full_like(q, float("nan"))
            B.amskv_append_attend(c.h, 0, i, k, v, q, o)
            assert B.amskv_status(c.h) == 0
            _check(o, q, ks, vs, range(i + 1), 1.0 / math.sqrt(D), i)


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_blocks_of_large_values(D, path):
    """Blocks whose power of two and bf16's least code exponent make more than one bf16 factor: |x| above 448 * 2^7."""
    sides, rows, heads = (3, 4, 12), 2, 2
    steps = _steps(rows, heads, sides, D, 3 * D)
    for i, (q, k, v) in enumerate(steps):
        q *= 2.0 ** -40
        k *= 2.0 ** (40 if i != 1 else 0)      # blocks of both kinds in one tile
        v[:, 0] *= 2.0 ** 60
    ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        for i, (q, k, v) in enumerate(steps):
            o = torch.full_like(q, float("nan"))
            B.amskv_append_attend(c.h, 0, i, k, v, q, o)
            assert B.amskv_status(c.h) == 0
            _check(o, q, ks, vs, range(i + 1), 1.0 / math.sqrt(D), i)


@pytest.mark.parametrize("path", ["rows", "tiles"])
def test_a_region_beyond_32_bits(path):
    """More than 2^32 codes, and inputs of more than 2^31 values: the first items, some in the middle, the last."""
    sides, rows, heads, D = (1, 2, 20), 2750, 16, 128
    g = torch.Generator(device="cuda").manual_seed(7)
    at = [0, 1373, 2749]
    ks, vs = [], []
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        assert B.amskv_cache_bytes(c.h)[0] > 1 << 32
        for i, s in enumerate(sides):
            q, k, v = (torch.randn(rows, heads, s * s, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(3))
            o = torch.full_like(q, float("nan"))
            B.amskv_append_attend(c.h, 0, i, k, v, q, o)
            assert B.amskv_status(c.h) == 0
            ks.append(ref.held_values(_np(k[at])))
            vs.append(ref.held_values(_np(v[at])))
            _check(o[at], q[at], ks, vs, range(i + 1), 1.0 / math.sqrt(D), i)
            assert not torch.isnan(o.view(-1, D)[::4097]).any()
        assert k.numel() > 1 << 31
        B.amskv_read_segment(c.h, 0, 2, q, o)
        assert (_np(q[at]) == ks[2]).all() and (_np(o[at]) == vs[2]).all()


def test_two_caches_on_two_streams():
    """Calls of two caches that overlap on the GPU give what they give one after the other."""
    sides, rows, heads, D = (2, 5, 12, 16), 3, 20, 64
    streams = [torch.cuda.Stream() for _ in range(2)]
    data = [_steps(rows, heads, sides, D, seed) for seed in (21, 22)]
    outs = [[[torch.empty_like(q) for q, _, _ in d] for d in data] for _ in range(2)]
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as a, Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as b:
        torch.cuda.synchronize()
        for n in range(2):
            for c in (a, b):
                B.amskv_cache_reset(c.h)
            for i in range(len(sides)):
                for j, c in enumerate((a, b)):
                    q, k, v = data[j][i]
                    B.amskv_append_attend(c.h, 0, i, k, v, q, outs[n][j][i], streams[j])
                    if n == 0:
                        streams[j].synchronize()
            torch.cuda.synchronize()
        assert B.amskv_status(a.h) == 0 and B.amskv_status(b.h) == 0
    for j in range(2):
        for x, y in zip(outs[0][j], outs[1][j]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("growth", [0.0, 15.0, 40.0])
@pytest.mark.parametrize("power", [88, -40])
def test_large_and_small_values_behind_a_maximum_that_grows(power, growth, path, D):
    """Logits near 0 in the first scale and near `growth` in the second."""
    sides, rows, heads = (8, 12), 2, 2
    steps = _steps(rows, heads, sides, D, 5 * D)
    for i, (q, k, v) in enumerate(steps):
        q *= 0.1
        q[..., 0], k[..., 0] = 1.0, (growth * math.sqrt(D) if i else 0.0)
        v *= 2.0 ** power
    ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        for i, (q, k, v) in enumerate(steps):
            o = torch.full_like(q, float("nan"))
            B.amskv_append_attend(c.h, 0, i, k, v, q, o)
            assert B.amskv_status(c.h) == 0
            _check(o, q, ks, vs, range(i + 1), 1.0 / math.sqrt(D), i)


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=["nan", "inf", "-inf"])
def test_a_block_with_a_number_that_is_none_or_an_infinity_is_no_number(bad, D, path):
    """It comes back as NaN in whole, its (row, head) attends to NaN, and nothing else changes; a clean append behind a reset
    leaves nothing of it."""
    sides, rows, heads = (3, 6, 9), 2, 3
    steps = _steps(rows, heads, sides, D, 31)
    scale = 1.0 / math.sqrt(D)
    ks, vs = ([ref.held_values(_np(x[i])) for x in steps] for i in (1, 2))
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])

        def run(data):
            outs = []
            B.amskv_cache_reset(c.h)
            for i, (q, k, v) in enumerate(data):
                outs.append(torch.zeros_like(q))
                B.amskv_append_attend(c.h, 0, i, k, v, q, outs[-1])
            assert B.amskv_status(c.h) == 0
            return outs

        plain = run(steps)
        for which in (1, 2):
            for tok in (0, 15, 17, 35):
                data = [[x.clone() for x in step] for step in steps]
                data[1][which][1, 2, tok, 5] = bad
                outs = run(data)
                back = [torch.zeros_like(steps[1][1]) for _ in range(2)]
                B.amskv_read_segment(c.h, 0, 1, *back)
                for n, want in ((0, ks[1]), (1, vs[1])):
                    want = torch.from_numpy(want).cuda().bfloat16()
                    if n + 1 == which:
                        want[1, 2, tok // 16 * 16:tok // 16 * 16 + 16] = float("nan")
                    assert torch.equal(torch.isnan(back[n]), torch.isnan(want)), (which, tok, n)
                    assert torch.equal(back[n].nan_to_num(), want.nan_to_num()), (which, tok, n)
                assert torch.equal(outs[0], plain[0])
                for i in (1, 2):
                    assert torch.isnan(outs[i][1, 2]).all(), (which, tok, i)
                    outs[i][1, 2] = plain[i][1, 2]
                    assert torch.equal(outs[i], plain[i]), (which, tok, i)
        for i, (q, _, _) in enumerate(steps):
            out = run(steps)[i]
            assert torch.equal(out, plain[i])
            _check(out, q, ks, vs, range(i + 1), scale, i)


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_a_path_of_ones_own_choice_depends_on_the_scale_alone(D, path):
    """Under every path but AUTO an image has the same outputs whatever other images it is computed with, bit for bit."""
    sides, heads = (1, 2, 4, 6, 10, 16), 5
    steps = _steps(60, heads, sides, D, 17)
    want = None
    for rows in (60, 2, 8, 30):
        with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
            B.amskv_set_attend_path(c.h, PATHS[path])
            outs = []
            for i, step in enumerate(steps):
                q, k, v = (x[:rows].contiguous() for x in step)
                outs.append(torch.zeros_like(q))
                B.amskv_append_attend(c.h, 0, i, k, v, q, outs[-1])
            assert B.amskv_status(c.h) == 0
        want = want or outs
        for i, (a, b) in enumerate(zip(outs, want)):
            assert torch.equal(a, b[:rows]), (rows, i)


@pytest.mark.parametrize("rows,heads,D,sides", [
    (2, 1, 64, (32, 2)),       # eight CTAs to the keys
    (16, 5, 64, (24, 5)),      # CTAs of two blocks, two to the keys
    (1, 5, 64, (5, 24)),       # eight warps, four CTAs to the keys
    (1, 1, 128, (22, 2)),
    (2, 1, 128, (32, 2)),
    (16, 5, 128, (13, 5)),     # two blocks, alone and two CTAs to the keys
    (8, 5, 128, (22, 5)),      # and four
    (4, 5, 128, (21, 9)),      # eight warps, two
    (2, 5, 128, (20, 11)),     # and four
])
def test_clusters_that_share_long_keys(rows, heads, D, sides):
    """Forms that only calls of few items under AUTO have."""
    test_a_schedule(rows, heads, D, sides, (0, 1, True), "auto")


@pytest.mark.parametrize("path", ["rows", "tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_errors_in_the_mean_are_those_of_two_roundings(D, path):
    """As for cross attention (0.85 * 2^-9 of the output, and of each probability before it meets its value), over the values the cache
    holds."""
    sides, rows, heads = (4, 9, 16), 2, 4
    g = torch.Generator(device="cuda").manual_seed(D)
    held, scale = [[], []], 1.0 / math.sqrt(D)
    with Cache(1, heads, D, rows, sides, [(0, 1, True)], flags=B.FLAG_KV_E4M3) as c:
        B.amskv_set_attend_path(c.h, PATHS[path])
        for i, s in enumerate(sides):
            q, k, v = (torch.randn(rows, heads, s * s, D, generator=g, device="cuda").bfloat16() for _ in range(3))
            out = torch.full_like(q, float("nan"))
            B.amskv_append_attend(c.h, 0, i, k, v, q, out)
            assert B.amskv_status(c.h) == 0
            for x, to in ((k, held[0]), (v, held[1])):
                to.append(torch.from_numpy(ref.held_values(_np(x))).cuda())
    kk, vv = (torch.cat(x, 2) for x in held)
    p = torch.softmax(scale * (q.double() @ kk.transpose(2, 3)), -1)
    want, spread_of_p = p @ vv, (p * p) @ (vv * vv)
    rms = float((out.double() - want).square().mean().sqrt())
    assert rms <= 2.0 ** -9 * float((want.square() + spread_of_p).mean().sqrt()), rms
