"""Rotary positions without a GPU: what the calls refuse, and the oracle's own identities."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2511_16047_b200 import binding as B

A = 1 << 20   # an aligned address that nothing reads: every call here is refused before any launch


def _refused(code, **change):
    args = dict(spec=B.make_rotary(64), table=A, table_rows=16, first=0, index=None, rows=2, T=4, head_dim=64, q_heads=2, Q=A,
                Q_out=2 * A, k_heads=2, K=3 * A, K_out=4 * A)
    args.update(change)
    with pytest.raises(B.AmskvError) as e:
        B.amskv_rotary(**args)
    assert e.value.code == code, (change, e.value)


@pytest.mark.parametrize("spec", [
    B.make_rotary(0), B.make_rotary(63), B.make_rotary(258), B.make_rotary(6, axes=2), B.make_rotary(64, axes=0),
    B.make_rotary(64, axes=4), B.make_rotary(64, layout=2), B.make_rotary(64, scaling=4), B.make_rotary(64, base=1.0),
    B.make_rotary(64, base=float("nan")), B.make_rotary(64, base=float("inf")), B.make_rotary(64, amplitude=-1.0),
    B.make_rotary(64, scaling=B.ROTARY_LINEAR, factor=0.5), B.make_rotary(64, scaling=B.ROTARY_LINEAR, factor=float("nan")),
    B.make_rotary(2, scaling=B.ROTARY_BASE, factor=2.0), B.make_rotary(64, scaling=B.ROTARY_BY_PARTS, factor=2.0),
    B.make_rotary(64, scaling=B.ROTARY_BY_PARTS, factor=2.0, original_length=100.0, beta_fast=1.0, beta_slow=1.0),
    B.make_rotary(64, scaling=B.ROTARY_BY_PARTS, factor=2.0, original_length=100.0, beta_slow=0.0)])
def test_bad_specs_are_refused(spec):
    with pytest.raises(B.AmskvError) as e:
        B.amskv_rotary_table_bytes(spec, 4)
    assert e.value.code == B.ERR_INVALID
    with pytest.raises(B.AmskvError) as e:
        B.amskv_rotary_table(spec, A, 4, A)
    assert e.value.code == B.ERR_INVALID
    _refused(B.ERR_INVALID, spec=spec)


@pytest.mark.parametrize("native", [True, False], ids=["native", "ctypes"])
def test_bad_arguments_are_refused(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_steps", None)
    for change in (dict(table=None), dict(table=A + 8), dict(table_rows=0), dict(rows=0), dict(T=0), dict(q_heads=0), dict(k_heads=-1),
                   dict(first=-1), dict(first=13), dict(Q=None), dict(Q=A + 2), dict(Q_out=None), dict(K_out=None), dict(K=None),
                   dict(k_heads=0), dict(index=A + 2), dict(index=A, index_row_stride=-1), dict(head_dim=56)):
        _refused(B.ERR_INVALID, **change)
    for change in (dict(head_dim=68), dict(head_dim=264), dict(rows=1 << 20, T=1 << 11, table_rows=1 << 11)):
        _refused(B.ERR_UNSUPPORTED, **change)
    for positions, count, table in ((None, 4, A), (A, 4, None), (A + 2, 4, A), (A, 4, A + 4), (A, 0, A)):
        with pytest.raises(B.AmskvError) as e:
            B.amskv_rotary_table(B.make_rotary(64), positions, count, table)
        assert e.value.code == B.ERR_INVALID
    # strides: an output that aliases itself, an input written to itself with other strides
    x = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16)
    _refused(B.ERR_INVALID, Q=x, Q_out=x[:1].expand(2, 2, 4, 64))
    y = torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16)
    _refused(B.ERR_INVALID, Q=y.transpose(1, 2), Q_out=y.data_ptr())
    with pytest.raises(AssertionError):
        B.amskv_rotary(B.make_rotary(64), A, 16, 0, torch.zeros(4, 2, dtype=torch.int32).t(), 2, 4, 64, 2, A, A)
    with pytest.raises(OverflowError):
        B.amskv_rotary(B.make_rotary(64), A, 16, 0, None, 1 << 40, 4, 64, 2, A, A)


@pytest.mark.skipif(torch.cuda.is_available(), reason="a device is there")
def test_without_a_device_the_calls_fail():
    _refused(B.ERR_CUDA)
    with pytest.raises(B.AmskvError) as e:
        B.amskv_rotary_table(B.make_rotary(64), A, 4, A)
    assert e.value.code == B.ERR_CUDA


def test_table_bytes():
    assert B.amskv_rotary_table_bytes(B.make_rotary(48, axes=2), 7) == 7 * 24 * 8


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes", [1, 2, 3])
def test_oracle_rotation_is_a_rotation_by_relative_positions(interleaved, axes):
    """Products of two rotated vectors depend on the difference of their positions only; the transpose undoes the rotation."""
    rng = np.random.default_rng(axes)
    dim = 12 * axes
    x, y = rng.standard_normal((2, 1, dim + 8))
    p, d = rng.integers(0, 50, (1, axes)).astype(float), rng.integers(0, 50, (1, axes)).astype(float)
    turn = lambda v, pos, **kw: ref.rotate(v, ref.rotary_angles(pos, dim), axes, interleaved, **kw)   # noqa: E731
    a = (turn(x, p) * turn(y, p + d)).sum()
    b = (turn(x, 0 * p) * turn(y, d)).sum()
    assert abs(a - b) < 1e-9
    assert np.abs(turn(turn(x, p), p, transposed=True) - x).max() < 1e-12
    assert (turn(x, p)[..., dim:] == x[..., dim:]).all()


@pytest.mark.skipif(B._steps is None, reason="the native module is not built")
def test_what_the_native_module_serves_and_what_it_leaves_to_ctypes():
    spec, x = B.make_rotary(64), torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16)
    good = [spec, A, 0, 0, None, None, 2, 4, 64, 2, x, x, 2, x.transpose(0, 1), x.data_ptr(), False, None]   # table_rows 0: refused by the library
    assert B._steps.rotary(*good) == B.ERR_INVALID
    idx = torch.zeros(2, 4, dtype=torch.int32)
    for at, value in ((4, idx), (4, idx[0]), (4, A), (5, 4), (15, True), (16, 0), (13, None)):
        assert B._steps.rotary(*good[:at], value, *good[at + 1:]) == B.ERR_INVALID, at
    for at, value in ((0, object()), (0, B.TokenBudget()), (4, idx.t()), (6, 1 << 31), (7, 4.0), (10, x.transpose(2, 3)), (15, 1), (2, "1")):
        assert B._steps.rotary(*good[:at], value, *good[at + 1:]) is None, at
    cross = [None, 0, 1, 7, x, x, x, x, None, None, 0, None]
    assert B._steps.cross_attend(*cross) == B.ERR_INVALID                                                      # no cache
    for at, value in ((8, idx[0]), (9, A), (11, 0), (4, A)):
        changed = cross[:at] + [value] + cross[at + 1:]
        assert B._steps.cross_attend(*changed) == B.ERR_INVALID or at == 4, at
    for at, value in ((1, 1.0), (3, 1 << 31), (5, x.transpose(0, 1)), (8, idx[:, ::2]), (0, 1.0)):
        assert B._steps.cross_attend(*cross[:at], value, *cross[at + 1:]) is None, at
    with pytest.raises(TypeError):
        B._steps.rotary(spec)


@pytest.mark.parametrize("native", [True, False], ids=["native", "ctypes"])
def test_lists_and_tables_that_the_kernels_would_misread(native, monkeypatch):
    """Of another type, with gaps, or too short: refused before the library is called.  What is right gets as far as the library, which
    here refuses something else (no launch can follow either way)."""
    if not native:
        monkeypatch.setattr(B, "_steps", None)
    spec, x = B.make_rotary(64, axes=2), torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)

    def rotary(table=A, index=None, rows=2, T=4, **kw):
        B.amskv_rotary(spec, table, 16, 0, index, rows, T, 60, 3, x, x, **kw)      # head_dim 60: below rotary_dim

    i32 = dict(dtype=torch.int32)
    for kw in (dict(table=torch.zeros(16, 32, 2)), dict(table=torch.zeros(20, 64)), dict(index=torch.zeros(4, **i32)), dict(index=torch.zeros(9, **i32)),
               dict(index=torch.zeros(2, 4, **i32)), dict(index=torch.zeros(3, 9, **i32)[:, 2:7]), dict(index=torch.zeros(1, 4, **i32), rows=1),
               dict(index=torch.zeros(1, 4, **i32).expand(2, 4)), dict(index=torch.zeros(8, **i32), index_row_stride=4),
               dict(index=torch.zeros(1, 4, **i32), index_row_stride=0), dict(index=torch.zeros(2, 5, **i32)[:, :4], index_row_stride=5),
               dict(index=torch.zeros(2, 4, 1, **i32)[:, :, 0].t()[:1].t(), T=1)):
        with pytest.raises(B.AmskvError) as e:
            rotary(**kw)
        assert e.value.code == B.ERR_INVALID, kw
    for kw in (dict(table=torch.zeros(16, 32, 2).double()), dict(table=torch.zeros(16, 64, 2)[:, ::2]), dict(table=torch.zeros(15, 32, 2)),
               dict(table=x), dict(index=torch.zeros(4, dtype=torch.int64)), dict(index=torch.zeros(4)), dict(index=torch.zeros(3, **i32)),
               dict(index=torch.zeros(0, **i32)), dict(index=torch.zeros(1, 4, **i32)), dict(index=torch.zeros(2, 3, **i32)),
               dict(index=torch.zeros(2, 4, dtype=torch.int16)), dict(index=torch.zeros(8, **i32), index_row_stride=5),
               dict(index=torch.zeros(2, 4, **i32), index_row_stride=8)):
        with pytest.raises(ValueError):
            rotary(**kw)
    for bad in (dict(first=1 << 63), dict(table_rows=1 << 63), dict(index=A, index_row_stride=1 << 63)):
        with pytest.raises(OverflowError):
            B.amskv_rotary(**{**dict(spec=spec, table=A, table_rows=16, first=0, index=None, rows=2, T=4, head_dim=60, q_heads=3, Q=A, Q_out=A), **bad})

    positions, table = torch.zeros(16, 2), torch.zeros(16, 32, 2)
    with pytest.raises(B.AmskvError) as e:
        B.amskv_rotary_table(B.make_rotary(64, axes=2, base=0.5), positions, 16, table)     # refused for its base
    assert e.value.code == B.ERR_INVALID
    for p, t in ((positions.double(), table), (positions.int(), table), (torch.zeros(2, 16).t(), table), (torch.zeros(16, 1).expand(16, 2), table),
                 (positions[:15], table), (torch.zeros(16, 3)[:, :2], table), (positions, table.double()), (positions, table[:15]),
                 (positions, torch.zeros(16, 64, 2)[:, ::2])):
        with pytest.raises(ValueError):
            B.amskv_rotary_table(spec, p, 16, t)
    with pytest.raises(OverflowError):
        B.amskv_rotary_table(spec, A, 1 << 64, A)


@pytest.mark.skipif(B._steps is None, reason="the native module is not built")
def test_keys_as_an_address_and_values_as_a_tensor():
    """Served where the tensor is contiguous, as an address is taken to be; refused where it is a view."""
    x = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16)
    for k, v in ((A, x), (x, A), (A, A)):
        assert B._steps.cross_attend(None, 0, 1, 7, k, v, x, x, None, None, 0, None) == B.ERR_INVALID      # no cache
    view = x.transpose(0, 1)
    for k, v in ((view, A), (A, view), (view, x)):
        assert B._steps.cross_attend(None, 0, 1, 7, k, v, x, x, None, None, 0, None) is None
        with pytest.raises(ValueError):
            B.amskv_cross_attend(None, 0, 1, 7, k, v, x, x)
