"""Pins of the few-token oracle: hand-worked codes, the format's invariants, the products against library routines, and
planted mistakes that the pins have to notice."""
import numpy as np
import pytest
import torch

from oracle import rom_few_oracle as F
from oracle import rom_oracle as O


def test_codes_worked_by_hand():
    # the largest is 12: scale 2, so |w| / s = 0 .25 .75 1.25 1.75 2.5 3.5 5 are the ties, and they go to even codes
    w = np.array([0.0, 0.5, 1.5, 2.5, 3.5, 5.0, 7.0, 10.0, 12.0, -0.5, -1.5, -12.0, 0.51, 1.49, 11.0, -0.0] + [0.0] * 16, np.float32)
    codes, scales = F.q4_quantize(w.reshape(1, 1, 32), 32)
    assert scales.ravel().tolist() == [2.0]
    assert codes.ravel()[:16].tolist() == [0, 0, 2, 2, 4, 4, 6, 6, 7, 0, 10, 15, 1, 1, 7, 0]
    assert F.q4_values(codes, scales, 32).ravel()[:12].tolist() == [0, 0, 2, 2, 4, 4, 8, 8, 12, 0, -2, -12]


def test_values_are_the_nearest_and_kept_by_a_second_pass():
    rng = np.random.default_rng(0)
    w = rng.standard_normal((2, 5, 136)).astype(np.float32)
    codes, scales = F.q4_quantize(w, 64)
    v = F.q4_values(codes, scales, 64)
    s = np.repeat(scales, 64, axis=2)[:, :, :136]
    every = np.concatenate([F.E2M1, -F.E2M1])
    assert np.allclose(np.abs(v - w), np.abs(w[..., None] - every * s[..., None]).min(-1), rtol=0, atol=1e-12)
    again = F.q4_quantize(v.astype(np.float32), 64)
    assert np.array_equal(F.q4_values(*again, 64), v)             # the largest is 6 s again


def test_groups_without_a_scale():
    w = np.ones((1, 1, 96), np.float32)
    w[0, 0, :32] = 0.0
    w[0, 0, 40] = np.inf
    w[0, 0, 70] = np.nan
    codes, scales = F.q4_quantize(w, 32)
    v = F.q4_values(codes, scales, 32)
    assert (v[0, 0, :32] == 0).all() and np.isnan(v[0, 0, 32:]).all()


def test_layout_places_every_weight_once():
    rng = np.random.default_rng(1)
    codes = rng.integers(1, 16, (2, 24, 136)).astype(np.uint8)
    scales = F.to_bf16(rng.uniform(0.5, 2, (2, 24, 5)).astype(np.float32))
    b = F.q4_layout(codes, scales, 32)
    assert b.size == 2 * 32 * 256 // 2 + 2 * 32 * 8 * 2
    nibbles = np.stack([b[:8192] & 15, b[:8192] >> 4])
    assert (nibbles > 0).sum() == codes.size and nibbles.sum(dtype=np.int64) == codes.sum(dtype=np.int64)
    # row 17, column 128 + 32 + 8 + 3 of the second matrix, by hand: matrix 1, tile 1, block 1, q 1, r 1, j 1, byte 1, high
    assert b[((1 * 2 + 1) * 2 + 1) * 1024 + (16 + 1) * 16 + 4 + 1] >> 4 == 0       # column 171 is past 136
    assert b[((1 * 2 + 1) * 2 + 0) * 1024 + (16 + 1) * 16 + 4 + 1] >> 4 == codes[1, 17, 32 + 8 + 3]


def test_products_against_library_routines():
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((6, 24)), rng.standard_normal((3, 16, 24))
    idx, gate = np.array([[0, 2]] * 3 + [[1, 1]] * 3), rng.uniform(0.1, 1, (6, 2))
    out, size = F.project(x, w, idx, gate)
    t = torch.from_numpy
    want = (torch.einsum("nkoi,ni->nko", t(w)[t(idx)], t(x)) * t(gate)[..., None]).sum(1)
    assert np.allclose(out, want.numpy()) and (size >= np.abs(out) - 1e-12).all()
    assert np.allclose(out[3:], F.project(x[3:], w, idx[3:, :1], gate[3:].sum(1, keepdims=True))[0])   # the same expert twice
    idx[0, 1] = 7
    assert np.allclose(F.project(x[:1], w, idx[:1], gate[:1])[0], F.project(x[:1], w, idx[:1, :1], gate[:1, :1])[0])
    scale, res = rng.standard_normal(6), rng.standard_normal((6, 16))
    assert np.allclose(F.project(x, w, idx, gate, scale, res)[0], F.project(x, w, idx, gate)[0] * scale[:, None] + res)


@pytest.mark.parametrize("pre_norm,skip", [(False, False), (True, True)])
def test_ffn_step_is_the_pinned_layer(pre_norm, skip):
    rng = np.random.default_rng(3)
    x, gu, down = rng.standard_normal((5, 24)), rng.standard_normal((4, 32, 24)), rng.standard_normal((4, 24, 16))
    idx = np.stack([rng.permutation(4)[:2] for _ in range(5)])
    gate = rng.uniform(0.1, 1, (5, 2))
    out, size, carried = F.ffn_step(x, gu, down, idx, gate, pre_norm, 1e-5, skip)
    want = O.ffn_moe_forward(x, gu, down, idx, gate, np.ones(24) if pre_norm else None, 1e-5, skip)
    assert np.allclose(out, want) and (size >= 0).all()
    # the third result bounds what a change of the pre-activations by a share of their terms does to the output
    wrong = F.ffn_step(x, gu * (1 + 1e-7 * np.sign(rng.standard_normal(gu.shape))), down, idx, gate, pre_norm, 1e-5, skip)[0]
    assert (np.abs(wrong - out) <= 1.01e-7 * carried + 1e-14).all()


@pytest.mark.parametrize("mistake", ["tie", "sign", "nibble", "scale", "gate"])
def test_planted_mistakes_are_noticed(mistake):
    rng = np.random.default_rng(4)
    w = rng.standard_normal((1, 16, 128)).astype(np.float32)
    w[0, 0, :2] = [6.0, 0.25]
    w[0, 0, 2:] = np.clip(w[0, 0, 2:], -5, 5)
    codes, scales = F.q4_quantize(w, 128)
    good = F.q4_layout(codes, scales, 128)
    x, idx, gate = rng.standard_normal((2, 128)), np.zeros((2, 1), int), np.full((2, 1), 0.5)
    if mistake == "tie":
        assert codes[0, 0, 1] == 0
        codes[0, 0, 1] = 1
    if mistake == "sign":
        codes ^= np.where(codes > 0, 8, 0).astype(np.uint8)
    if mistake == "nibble":
        codes = codes.reshape(1, 16, 64, 2)[..., ::-1].reshape(1, 16, 128)
    if mistake == "scale":
        scales = np.roll(scales, 1, axis=1)
    if mistake == "gate":
        v = F.q4_values(codes, scales, 128)
        assert not np.allclose(F.project(x, v, idx, gate)[0], F.project(x, v, idx)[0])
        return
    assert not np.array_equal(F.q4_layout(codes, scales, 128), good)
