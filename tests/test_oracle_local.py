"""Pins of the 64-bit forms of the local-gradient operators (CPU only): the
e4m3 table against torch's type, the checkpoint's error bound, and the
gradients against differences."""
import numpy as np
import torch

from oracle import local as ol


def test_e4m3_table_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = ol.e4m3_table()
    assert np.array_equal(got, want, equal_nan=True)


def test_e4m3_nearest_rounds_like_torch():
    rng = np.random.default_rng(0)
    z = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.02, 4000),
                        ol.e4m3_table()[:0x7F], [0.0, -0.0]])
    pos = ol.e4m3_table()[:0x7F]
    z = np.concatenate([z, (pos[1:] + pos[:-1]) / 2]).astype(np.float32)  # ties
    want = torch.from_numpy(z).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ol.e4m3_nearest(z.astype(np.float64)), want)


def test_pack_error_bound_and_scale():
    rng = np.random.default_rng(1)
    x = rng.normal(0, 1, (64, 70)) * np.exp2(rng.integers(-140, 100, (64, 70)))
    q, s = ol.pack(x)
    y = ol.unpack(q, s)
    k = np.repeat(s.astype(int) - 127, 32, axis=1)[:, :70]
    bound = np.maximum(np.abs(x) / 16, np.exp2(k - 10.0))
    assert (np.abs(y - x) <= bound).all()
    assert k.min() >= ol.MIN_EXP
    # the scale is the smallest that holds the group: half of it would not
    top = np.abs(x[:, :32]).max(1)
    k0 = s[:, 0].astype(int) - 127
    assert (top <= 448 * np.exp2(k0 * 1.0)).all()
    assert ((top > 448 * np.exp2(k0 - 1.0)) | (k0 == ol.MIN_EXP)).all()


def test_pack_borders():
    x = np.zeros((4, 3))
    x[1] = [448.0, 1.0, -448.0]
    x[2] = [np.nextafter(np.float32(448), np.float32(500)), 1.0, 0.0]
    x[3] = [np.inf, -np.nan, 3.5]
    q, s = ol.pack(x)
    assert list(s[:, 0]) == [10, 127, 128, 120]
    assert list(q[0]) == [0, 0, 0] and list(q[1]) == [0x7E, 0x38, 0xFE]
    assert list(q[3]) == [0x7F, 0x7F, 0x7E]


def test_gradients_against_differences():
    rng = np.random.default_rng(2)
    tokens = np.array([4, 7, 4, -1, 11, 7, 4])
    table, c = rng.normal(size=(6, 5)), rng.normal(size=(7, 5))
    loss = lambda tb: (c * ol.embed(tokens, tb, 3, 1.5)).sum()
    grad, count, _ = ol.embed_grad(tokens, c, 6, 3, 1.5)
    assert list(count) == [0, 3, 0, 0, 2, 0]
    for r in range(6):
        e = np.zeros_like(table)
        e[r, 2] = 0.5
        assert abs(loss(table + e) - loss(table - e) - grad[r, 2]) < 1e-12
    x, w, dy = rng.normal(size=(9, 4)), rng.normal(size=(3, 4)), rng.normal(size=(9, 3))
    g, _ = ol.wgrad(dy, x, 2.0)
    loss = lambda w: 2.0 * (dy * (x @ w.T)).sum()
    e = np.zeros_like(w)
    e[1, 3] = 0.5
    assert abs(loss(w + e) - loss(w - e) - g[1, 3]) < 1e-12
