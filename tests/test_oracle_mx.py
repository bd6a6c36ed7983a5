"""Pins of the block-scaled oracle: code tables, scales and roundings worked out by hand, the packed layout, and the
operators against torch in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx as X


def test_code_tables():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(X.E4M3, t, equal_nan=True)
    assert X.E2M1.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]


@pytest.mark.parametrize("bits,amax,byte", [
    (8, 448.0, 127), (8, 449.0, 128), (8, 224.0, 126), (8, 1.0, 127 - 8), (8, 1.75, 127 - 8), (8, 1.76, 127 - 7),
    (8, 0.0, 0), (8, 1e-45, 0), (8, 2.0 ** -119, 0), (8, 3.0e38, 127 + 120), (8, np.inf, 255), (8, np.nan, 255),
    (4, 6.0, 127), (4, 6.01, 128), (4, 3.0, 126), (4, 4.0, 127), (4, 0.02, 127 - 8), (4, np.inf, 255)])
def test_scale_bytes(bits, amax, byte):
    x = np.zeros((1, 32))
    x[0, 5] = -amax
    codes, s = X.quantize(x, bits)
    assert codes.shape == (1, 128) and s.tolist() == [[byte, 0, 0, 0]]
    if byte == 255:
        assert np.isnan(X.dequantize(codes, s, bits, 32)).all()


def test_roundings():
    # scale 1 (a 6 and a 448 in the block); ties go to the even code
    x = np.zeros((1, 32))
    x[0, :9] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.26]
    assert X.requantized(x, 4)[0, :9].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -.5]
    x[0, :6] = [448, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -9]
    assert X.requantized(x, 8)[0, :6].tolist() == [448, 16, 20, 0, 2 * 2.0 ** -9, -2.0 ** -9]


def test_quantiser_against_torch_and_itself():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(40, 200)) * np.exp(rng.normal(size=(40, 1)) * 5)
    codes, s = X.quantize(x, 8)
    v = np.pad(x, ((0, 0), (0, 56))).reshape(40, -1, 32) / 2.0 ** (s.astype(float) - 127)[..., None]
    assert np.abs(v).max() <= 448 and (np.abs(v).max(axis=-1) > 224)[:, :6].all()
    t = torch.from_numpy(v).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (t.reshape(40, -1) != codes).mean() < 1e-4      # (torch rounds twice, by way of 32 bits)
    for bits in (4, 8):
        q = X.requantized(x, bits)
        assert np.array_equal(X.requantized(q, bits), q)   # block-scaled numbers keep their values
        # half a step: E4M3 2^-4 of the value or half of 2^-9 of the scale, E2M1 2^-2 and half of 0.5
        scale = np.repeat(2.0 ** (X.quantize(x, bits)[1].astype(float) - 127), 32, axis=1)[:, :200]
        assert (np.abs(q - x) <= np.maximum(np.abs(x) * (2.0 ** -4 if bits == 8 else 2.0 ** -2), scale * (2.0 ** -10 if bits == 8 else 0.25))).all()


def test_packed_layout_by_hand():
    codes = np.zeros((17, 256), dtype=np.uint8)
    scales = np.zeros((17, 8), dtype=np.uint8)
    codes[16, 128 + 32 * 2 + 5] = 9
    scales[16, 6] = 77
    b, s = X.pack_weight(codes, scales, 4)
    assert b.size == 2 * 2 * 1024 and s.size == 2 * 256
    # tile (1, 1), lane 16 * 2 + 0, byte 2, high nibble (column 5)
    assert np.flatnonzero(b).tolist() == [3 * 1024 + 32 * 16 + 2] and b.max() == 9 << 4
    assert np.flatnonzero(s).tolist() == [256 + 32 * 4 + 1]
    b, _ = X.pack_weight(codes, scales, 8)
    # column 69 of the tile: half 1, piece 0, byte 5
    assert b.size == 2 * 2 * 2048 and np.flatnonzero(b).tolist() == [3 * 2048 + 1024 + 0 * 16 + 5]


def test_expert_and_ffn_against_torch():
    rng = np.random.default_rng(1)
    x, (w1, w3), w2 = rng.normal(size=(5, 64)), rng.normal(size=(2, 96, 64)), rng.normal(size=(64, 96))
    t = [torch.from_numpy(v) for v in (x, w1, w3, w2)]
    h = torch.nn.functional.silu(t[0] @ t[1].T) * (t[0] @ t[2].T)
    y = X.expert(x, w1, w3, w2)
    assert np.allclose(y, X.requantized(h.numpy()) @ w2.T, rtol=1e-12, atol=1e-12)
    assert np.linalg.norm(y - (h @ t[3].T).numpy()) < 2.0 ** -4 * np.linalg.norm(y)
    # a token that names one expert twice takes it twice; an absent expert adds nothing; the shared one is gated
    ids, w = np.array([[0, 0], [0, 1], [2, 0], [1, 1], [2, 2]]), rng.random((5, 2))
    m = {0: (w1, w3, w2), 1: (w3, w1, w2)}
    got = X.moe_ffn(x, ids, w, m, [(w1, w1, w2)], gate := rng.normal(size=64))
    for n in range(5):
        ref = sum((w[n, j] * X.expert(x[n:n + 1], *m[ids[n, j]])[0] for j in range(2) if ids[n, j] in m), np.zeros(64))
        ref = ref + X.expert(x[n:n + 1], w1, w1, w2)[0] / (1 + np.exp(-x[n] @ gate))
        assert np.allclose(got[n], ref, rtol=1e-12, atol=1e-12)
