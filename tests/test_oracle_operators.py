"""The 64-bit definitions against independent forms of them."""
import numpy as np
import pytest
import torch

from oracle import operators as ref


def test_e4m3_rounding_is_that_of_the_type():
    x = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 20000), np.exp2(np.random.default_rng(1).uniform(-12, 8.8, 20000)),
                        np.arange(0, 256) / 4096.0, [0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert (ref.round_e4m3(x.astype(np.float64)) == want).all()


@pytest.mark.parametrize("T", [1, 15, 16, 17, 40])
def test_held_values_are_near_and_exact_in_bf16(T):
    rng = np.random.default_rng(T)
    x = rng.standard_normal((2, 3, T, 8)) * np.exp2(rng.integers(-30, 30, (2, 3, 1, 1)))
    x[0, 0] = 0.0
    y = ref.held_values(x)
    e = np.repeat(ref.held_exponents(x), 16, -1)[..., :T, None]
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * np.exp2(e))).all()
    assert (torch.from_numpy(y).bfloat16().double().numpy() == y).all()
    assert (ref.held_exponents(x)[0, 0] == 0).all()
    top = np.abs(x[1, 1, :16]).max()
    e0 = ref.held_exponents(x)[1, 1, 0]
    assert 448 * 2.0 ** (e0 - 1) < top <= 448 * 2.0 ** e0


def test_attention_is_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 5, 16)), rng.standard_normal((3, 9, 16)), rng.standard_normal((3, 9, 16))
    out, size = ref.attention(q, k, v, 0.3)
    t = [torch.from_numpy(x) for x in (q, k, v)]
    want = torch.softmax(0.3 * t[0] @ t[1].transpose(1, 2), -1) @ t[2]
    assert np.abs(out - want.numpy()).max() < 1e-12
    assert (size >= np.abs(out) - 1e-12).all()
    assert (ref.attention(q, k[:, :0], v[:, :0], 0.3)[0] == 0).all()
