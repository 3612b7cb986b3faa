"""Pins for the oracle's 8-bit cache (oracle/kv8.py) and rotary positions (oracle/rotary.py): the format against torch's own type,
blocks and scales against a worked case, rotations against the half-pairing rope and what the scalings promise."""
import math

import numpy as np
import pytest
import torch

from oracle import forward as ofwd, kv8, rotary


def test_values_are_those_of_torchs_e4m3():
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.VALUES, t, equal_nan=True)


def test_encoding_rounds_as_torch_does_ties_included():
    rng = np.random.default_rng(1)
    up = kv8.VALUES[:127]
    ties = (up[1:] + up[:-1]) / 2
    x = np.concatenate([rng.normal(0, 1, 5000) * 2.0 ** rng.integers(-12, 8, 5000), ties, -ties, up, -up, ties * (1 + 2.0 ** -20)])
    x = np.float32(np.clip(x, -448, 448)).astype(np.float64)
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv8.encode(x), want)
    assert kv8.decode(kv8.encode([500.0, -1e9])).tolist() == [448.0, -448.0]
    assert np.isnan(kv8.decode(kv8.encode([np.inf, -np.inf, np.nan]))).all()


def test_scales():
    assert kv8.scale_for([448.0]) == 1.0 and kv8.scale_for([448.0001]) == 2.0 and kv8.scale_for([224.0]) == 0.5
    assert kv8.scale_for([0.0]) == 2.0 ** -40 == kv8.scale_for([np.nan, np.inf]) and kv8.scale_for([1e30]) == 2.0 ** 40
    assert kv8.scale_for([np.inf, -3.0]) == kv8.scale_for([3.0])


def test_a_blocks_scale_grows_with_its_tokens_and_starts_anew():
    p = kv8.Plane(128, 2)
    p.append(0, [[1.0, -1.75], [0.5, 0.01]])                 # 1.75 = 448 * 2^-8
    assert p.scale[0] == 2.0 ** -8 and p.numbers(2)[0].tolist() == [1.0, -1.75]
    small = p.numbers(2)[1, 1]
    p.append(2, [[100.0, 0.0]])                              # the scale grows to 2^-2: 0.01 / 2^-2 = 0.04 is still a normal code
    assert p.scale[0] == 2.0 ** -2 and p.numbers(3)[1, 1] == small and p.numbers(3)[0].tolist() == [1.0, -1.75]
    p.append(3, [[400.0 * 256, 0.0]])                        # 2^8: 0.01 is below half of the smallest step, 2^-9 * 2^8
    assert p.scale[0] == 2.0 ** 8 and p.numbers(4)[1, 1] == 0.0 and p.numbers(4)[0, 0] == 1.0
    p.append(2, [[1.0, 1.0]])                                # rolled back to two tokens: the scale stays
    assert p.scale[0] == 2.0 ** 8
    p.append(0, [[1.0, 1.0]])                                # ... and starts anew with the block's first token
    assert p.scale[0] == 2.0 ** -8
    p.append(63, [[2.0, 2.0], [1e-3, 0.0]])                  # over the border: two blocks, two scales
    assert p.scale[0] == 2.0 ** -7 and p.scale[1] == kv8.scale_for([1e-3])


def test_plain_rotary_positions_are_the_half_pairing_rope():
    rng = np.random.default_rng(2)
    x, pos = rng.normal(size=(5, 3, 64)), np.array([0, 1, 7, 1000, 123456])
    f = rotary.frequencies(64, 1e4)
    want = ofwd.rope(x, pos, 1e4)
    assert np.allclose(rotary.turn(x, pos, f), want, atol=1e-9)
    # interleaved is the same with the entries in another order
    order = np.arange(64).reshape(2, 32).T.reshape(-1)       # place 2i holds entry i, 2i + 1 entry i + 32
    assert np.allclose(rotary.turn(x[..., order], pos, f, interleaved=True), want[..., order], atol=1e-9)
    # part of the head
    y = rotary.turn(x, pos, rotary.frequencies(16, 1e4))
    assert np.array_equal(y[..., 16:], x[..., 16:]) and np.allclose(y[..., :16], ofwd.rope(x[..., :16], pos, 1e4), atol=1e-9)
    assert np.allclose(rotary.turn(x, pos, f, magnitude=1.5), 1.5 * want, atol=1e-9)


@pytest.mark.parametrize("interleaved", [False, True])
def test_products_of_rotated_rows_depend_on_the_distance_alone(interleaved):
    rng = np.random.default_rng(3)
    q, k = rng.normal(size=(1, 1, 32)), rng.normal(size=(1, 1, 32))
    f = rotary.frequencies(24, 5e5, "parts", 8.0, 1.0, 4.0, 512)
    dots = [float((rotary.turn(q, [p + 11], f, interleaved) * rotary.turn(k, [p], f, interleaved)).sum()) for p in (0, 5, 4000)]
    assert np.allclose(dots, dots[0], atol=1e-9)


def test_scalings():
    plain = rotary.frequencies(32, 1e4)
    assert np.allclose(rotary.frequencies(32, 1e4, "linear", 4.0), plain / 4)
    base = rotary.frequencies(32, 1e4, "base", 4.0)
    assert base[0] == plain[0] and np.isclose(base[-1], plain[-1] / 4)
    assert np.allclose(base, (1e4 * 4.0 ** (32 / 30)) ** (-np.arange(16) / 16))
    parts = rotary.frequencies(32, 1e4, "parts", 8.0, 1.0, 4.0, 2048)
    turns = 2048 * plain / (2 * math.pi)
    assert np.allclose(parts[turns > 4], plain[turns > 4]) and np.allclose(parts[turns < 1], plain[turns < 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all((parts[mid] < plain[mid]) & (parts[mid] > plain[mid] / 8)) and np.all(np.diff(parts) < 0)


def test_a_forward_on_the_8_bit_cache_stays_near_the_exact_one():
    from paper_2510_26527_amd import synth
    shape = synth.Shape(2, 128, 4, 2, 64, 256, 97)
    w = synth.make_weights(shape, 3, torch.float32, std=0.08)
    cfg = ofwd.ModelConfig(**shape.asdict())
    toks = synth.make_tokens(shape.vocab, (2, 70), 5)
    exact, eight = ofwd.KVCache(cfg, 2, 128), kv8.KVCache8(cfg, 2, 128)
    a, b = ofwd.forward(cfg, w, toks, exact), ofwd.forward(cfg, w, toks, eight)
    off = np.abs(a - b).max() / np.abs(a).max()
    assert 0 < off < 0.1                                      # each K and V entry is off by up to 2^-4 of itself
    # rows one at a time read the same codes where no scale grew, so they stay as near
    eight.truncate([60, 60])
    c = np.concatenate([ofwd.forward(cfg, w, toks[:, r:r + 1], eight) for r in range(60, 70)], axis=1)
    assert np.abs(c - a[:, 60:]).max() / np.abs(a).max() < 0.1
