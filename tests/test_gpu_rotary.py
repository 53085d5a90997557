"""Rotary positions on the GPU against the definition in 64 bits.

Tolerances.  A table entry: the angle, rounded twice, is right to 2^-23 of at most pi / 4, the sums to two units of 2^-24, the
amplitude's product to one more: under 2^-21.  An output: three fp32 roundings of |u| + |w| times the amplitude
and the table's error times the same, under 2^-20 of it together, then half a step of bf16, 2^-8 of the value."""
import decimal
from decimal import Decimal

import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2511_16047_b200 import binding as B

pytestmark = pytest.mark.gpu

SCALINGS = {"plain": (B.ROTARY_PLAIN, {}), "linear": (B.ROTARY_LINEAR, {"factor": 3.5}), "base": (B.ROTARY_BASE, {"factor": 8.0}),
            "parts": (B.ROTARY_BY_PARTS, {"factor": 4.0, "original_length": 680.0})}


def _spec(dim, axes, interleaved, scaling, **kw):
    code, extra = SCALINGS[scaling]
    return (B.make_rotary(dim, axes=axes, layout=B.ROTARY_INTERLEAVED if interleaved else B.ROTARY_HALF, scaling=code, **extra, **kw),
            dict(extra, scaling=scaling))


def _amplitude(scaling):
    return 1.0 + 0.1 * np.log(4.0) if scaling == "parts" else 1.0


def _table(spec, dim, positions):
    """With guard rows behind it, which have to stay as they are."""
    n = positions.shape[0]
    assert B.amskv_rotary_table_bytes(spec, n) == n * dim * 4
    t = torch.full((n + 2, dim // 2, 2), 7.0, device="cuda")
    B.amskv_rotary_table(spec, positions, n, t)
    assert (t[n:] == 7.0).all()
    return t


@pytest.mark.parametrize("scaling", sorted(SCALINGS))
@pytest.mark.parametrize("dim,axes,count", [(64, 1, 1), (128, 1, 1000), (256, 1, 37), (48, 2, 333), (12, 3, 5), (96, 3, 257), (4, 1, 100000)])
def test_table(dim, axes, count, scaling):
    g = torch.Generator().manual_seed(dim + count)
    pos = torch.randint(0, 1 << 20, (count, axes), generator=g).float()
    pos[::3] *= 0.37          # fractions
    pos[::5] = -pos[::5]
    spec, kw = _spec(dim, axes, False, scaling)
    got = _table(spec, dim, pos.cuda())[:count].cpu().double().numpy()
    angle = ref.rotary_angles(pos.numpy(), dim, **kw)
    amp = _amplitude(scaling)
    want = np.stack([np.cos(angle), np.sin(angle)], -1) * amp
    assert np.abs(got - want).max() <= 2.0 ** -21 * amp


def test_table_of_far_positions_and_a_given_amplitude():
    pos = torch.tensor([[0.0], [1.0], [2.0 ** 24], [2.0 ** 31], [1e15]])
    spec = B.make_rotary(64, amplitude=0.5)
    got = _table(spec, 64, pos.cuda())[:5].cpu().double().numpy()
    angle = ref.rotary_angles(pos.numpy(), 64)
    want = np.stack([np.cos(angle), np.sin(angle)], -1) * 0.5
    # fp64 angles on both sides: off by 2^-52 of the angle
    tol = 2.0 ** -22 + 0.5 * np.abs(angle)[..., None] * 2.0 ** -51
    assert (np.abs(got - want) <= tol)[:4].all()
    assert np.abs(np.linalg.norm(got, axis=-1) - 0.5).max() < 1e-6   # (at 10^15 the angle is lost, not the length)


def test_table_of_no_numbers_and_of_the_smallest():
    pos = torch.tensor([[float("nan")], [float("inf")], [-float("inf")], [1e-45], [-3e-39], [1.17549435e-38], [-0.0]])
    got = _table(B.make_rotary(8), 8, pos.cuda())[:7].cpu()
    assert torch.isnan(got[:3]).all()
    assert (got[3:, :, 0] == 1.0).all() and (got[3:, :, 1].abs() <= 2.0 ** -30).all()


def _views(x):
    """The same values behind other strides: heads innermost but one, as a projection leaves them."""
    r, h, t, d = x.shape
    y = torch.zeros(r, t, h + 1, d + 8, dtype=x.dtype, device=x.device)
    v = y[:, :, 1:, :d].transpose(1, 2)
    v.copy_(x)
    return v


def _check(got, x, angles, axes, interleaved, amp, transposed, what):
    x64 = x.cpu().double().numpy()
    want = ref.rotate(x64, angles, axes, interleaved, amp, transposed)
    size = np.zeros_like(x64)
    pairs = ref.rotary_pairs(2 * angles.shape[-1], axes, interleaved)
    both = np.abs(x64[..., pairs[:, 0]]) + np.abs(x64[..., pairs[:, 1]])
    size[..., pairs[:, 0]], size[..., pairs[:, 1]] = both, both
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * amp * size
    err = np.abs(got.cpu().double().numpy() - want)
    assert (err <= tol).all(), (what, (err - tol).max())


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,kv,T,D,dim,axes,scaling", [
    (1, 1, 1, 1, 64, 64, 1, "plain"),
    (2, 16, 16, 1, 64, 64, 1, "plain"),
    (2, 3, 1, 25, 64, 64, 2, "linear"),
    (3, 5, 2, 169, 64, 48, 1, "parts"),
    (2, 4, 4, 100, 128, 128, 1, "base"),
    (2, 8, 2, 256, 128, 128, 2, "plain"),
    (1, 2, 2, 33, 128, 20, 1, "plain"),       # pairs that no 16-byte piece holds
    (2, 2, 1, 17, 72, 12, 3, "plain"),
    (1, 3, 3, 9, 8, 2, 1, "plain"),
    (1, 2, 1, 50, 256, 256, 1, "plain"),
    (2, 1, 1, 7, 128, 96, 3, "parts"),
    (37, 30, 30, 36, 64, 64, 1, "plain"),
])
def test_rotation(rows, heads, kv, T, D, dim, axes, scaling, interleaved):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + T)
    q, k = (torch.randn(rows, h, T, D, generator=g, device="cuda").bfloat16() for h in (heads, kv))
    spec, kw = _spec(dim, axes, interleaved, scaling)
    n = T + 13
    pos = torch.rand(n, axes, generator=g, device="cuda") * 1000
    table = _table(spec, dim, pos)
    angles, amp = ref.rotary_angles(pos.cpu().numpy(), dim, **kw), _amplitude(scaling)

    # token numbers from 5 on, contiguous tensors
    qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    B.amskv_rotary(spec, table, n, 5, None, rows, T, D, heads, q, qo, kv, k, ko)
    for got, x in ((qo, q), (ko, k)):
        _check(got, x, angles[5:5 + T], axes, interleaved, amp, False, "contiguous")

    # the transpose, of views into views
    qv, kk = _views(q), _views(k)
    qo2, ko2 = _views(torch.zeros_like(q)), _views(torch.zeros_like(k))
    B.amskv_rotary(spec, table, n, 0, None, rows, T, D, heads, qv, qo2, kv, kk, ko2, transposed=True)
    for got, x in ((qo2, q), (ko2, k)):
        _check(got, x, angles[:T], axes, interleaved, amp, True, "transposed views")
    assert (qo2._base[:, :, 0] == 0).all() and (qo2._base[..., D:] == 0).all()   # nothing beside the view is written

    # rows of their own, some without a position or outside the table; in place
    index = torch.randint(0, n, (rows, T + 3), generator=g, device="cuda", dtype=torch.int32)
    index[:, ::4] = -1
    index[0, 0] = n                   # behind the last row of the table (whose guard rows hold 7)
    index[-1, T // 2] = -2 ** 31
    index = index[:, :T]
    idx = index.cpu().numpy()
    inside = (idx >= 0) & (idx < n)
    per_row = np.where(inside[..., None], angles[np.where(inside, idx, 0)], np.nan)[:, None]
    qi, ki = q.clone(), k.clone()
    B.amskv_rotary(spec, table, n, 0, index, rows, T, D, heads, qi, qi, kv, ki, ki)
    for got, x in ((qi, q), (ki, k)):
        _check(got, x, np.broadcast_to(per_row, (*x.shape[:3], dim // 2)), axes, interleaved, amp, False, "in place")
    # one list of rows for all, Q alone
    qo.fill_(9.0)
    B.amskv_rotary(spec, table, n, 0, index[0].contiguous(), rows, T, D, heads, q, qo)
    _check(qo, q, np.broadcast_to(per_row[:1], (*q.shape[:3], dim // 2)), axes, interleaved, amp, False, "one index")


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
def test_the_transpose_is_the_gradient(interleaved):
    """Against differences: the rotation is linear, so <y(x + h e) - y(x), g> / h is its gradient in direction e exactly but for
    the roundings of the outputs."""
    T, D = 6, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    spec, _ = _spec(D, 1, interleaved, "parts")
    table = _table(spec, D, torch.arange(T, device="cuda").float()[:, None].contiguous())
    x, e, up = (torch.randn(1, 1, T, D, generator=gen, device="cuda").bfloat16() for _ in range(3))
    y0, y1, grad = (torch.empty_like(x) for _ in range(3))
    xe = (x.float() + 4.0 * e.float()).bfloat16()
    B.amskv_rotary(spec, table, T, 0, None, 1, T, D, 1, x, y0)
    B.amskv_rotary(spec, table, T, 0, None, 1, T, D, 1, xe, y1)
    B.amskv_rotary(spec, table, T, 0, None, 1, T, D, 1, up, grad, transposed=True)
    up64, step = up.double(), xe.double() - x.double()
    by_difference = float(((y1.double() - y0.double()) * up64).sum())
    by_gradient = float((grad.double() * step).sum())
    tol = 2.0 ** -8 * float(((y0.abs() + y1.abs()).double() * up64.abs()).sum() + (grad.double().abs() * step.abs()).sum())
    assert abs(by_difference - by_gradient) <= 1.02 * tol


def test_captured_and_on_another_stream():
    T, D, heads, rows = 64, 64, 4, 2
    spec, kw = _spec(D, 2, False, "plain")
    pos = torch.rand(T, 2, device="cuda") * 64
    x, out = torch.randn(rows, heads, T, D, device="cuda").bfloat16(), torch.zeros(rows, heads, T, D, device="cuda").bfloat16()
    table = torch.zeros(T, D // 2, 2, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def calls():
        B.amskv_rotary_table(spec, pos, T, table, side)
        B.amskv_rotary(spec, table, T, 0, None, rows, T, D, heads, x, out, stream=side)

    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    x.copy_(torch.randn(rows, heads, T, D, device="cuda"))
    pos.copy_(torch.rand(T, 2, device="cuda") * 64)
    graph.replay()
    torch.cuda.synchronize()
    _check(out, x, ref.rotary_angles(pos.cpu().numpy(), D, **kw), 2, False, 1.0, False, "replayed")


@pytest.mark.parametrize("in_place", [False, True], ids=["out of place", "in place"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,T,D,dim", [(2, 3, 9, 64, 64), (37, 30, 36, 64, 48), (2, 2, 7, 128, 20)])
def test_a_token_without_a_position_is_passed_on_bit_for_bit(rows, heads, T, D, dim, interleaved, in_place):
    """Whatever its channels hold: infinities, numbers that are none, zeros with a sign."""
    gen = torch.Generator(device="cuda").manual_seed(dim)
    bits = torch.randint(-2 ** 15, 2 ** 15, (rows, heads, T, D), generator=gen, device="cuda", dtype=torch.int32).to(torch.int16)
    bits[..., ::3], bits[..., 1::5], bits[..., 2::7] = 0x7f80, -0x8000, 0x7fc1      # infinity, -0, no number
    spec, _ = _spec(dim, 1, interleaved, "plain")
    table = _table(spec, dim, torch.arange(4, device="cuda").float()[:, None].contiguous())
    index = torch.full((rows, T), -1, dtype=torch.int32, device="cuda")
    index[:, ::2] = 4
    for transposed in (False, True):
        x = bits.clone().view(torch.bfloat16)
        out = x if in_place else torch.zeros_like(x)
        B.amskv_rotary(spec, table, 4, 0, index, rows, T, D, heads, x, out, transposed=transposed)
        assert torch.equal(out.view(torch.int16), bits)


def _exact_entries(positions, dim, base):
    """Cosines and sines by decimal arithmetic of 90 digits, and the angles."""
    with decimal.localcontext() as ctx:
        ctx.prec = 90
        pi = sum((Decimal(4) / (8 * n + 1) - Decimal(2) / (8 * n + 4) - Decimal(1) / (8 * n + 5) - Decimal(1) / (8 * n + 6)) / 16 ** n for n in range(75))
        out, angles = np.empty((len(positions), dim // 2, 2)), np.empty((len(positions), dim // 2))
        for i in range(dim // 2):
            w = (Decimal(-2 * i) / dim * Decimal(base).ln()).exp()
            for n, p in enumerate(positions):
                angle = Decimal(p) * w
                rest = float(angle - 2 * pi * (angle / (2 * pi)).to_integral_value())
                out[n, i], angles[n, i] = (np.cos(rest), np.sin(rest)), float(angle)
        return out, angles


@pytest.mark.parametrize("dim,base", [(64, 10000.0), (128, 500000.0), (12, 3.0)])
def test_far_positions_against_many_digits(dim, base):
    """To what the header promises: 2^-31 of a turn, 2^-50 of the angle and 2^-64 of a turn per unit of position, and an entry's own
    2^-21."""
    pos = torch.tensor([[1.0], [0.3], [8191.25], [1e6], [2.0 ** 23 - 0.5], [2.0 ** 24 + 2], [-2.0 ** 28 - 32], [2.0 ** 31], [1e11], [-7e12], [1e15]])
    got = _table(B.make_rotary(dim, base=base), dim, pos.cuda())[:len(pos)].cpu().double().numpy()
    want, angles = _exact_entries([float(p) for p in pos[:, 0]], dim, base)
    at = pos[:, :1].abs().double().numpy()
    tol = 2.0 ** -21 + 2 * np.pi * (2.0 ** -31 + at * 2.0 ** -64) + np.abs(angles) * 2.0 ** -50
    assert (np.abs(got - want) <= tol[..., None]).all()
    assert (tol[:9] < 2e-4).all()
