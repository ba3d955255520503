"""Pins of the oracle's decode-step operators against closed forms and worked numbers (CPU)."""
import numpy as np
import pytest

from oracle import decode


def test_rms_norm_closed_forms():
    x = np.array([[3.0, -4.0]])
    h, v = decode.rms_norm(x, None, np.ones(2), 0.0, 0.0)
    assert np.array_equal(h, x)
    np.testing.assert_allclose(v, x / np.sqrt(12.5), rtol=1e-15)
    h, v = decode.rms_norm(x, np.array([[1.0, 4.0]]), np.array([1.0, 2.0]), 1.0, 0.0)
    np.testing.assert_allclose(h, [[4.0, 0.0]])
    np.testing.assert_allclose(v, [[4 / np.sqrt(8) * 2, 0.0]], rtol=1e-15)
    assert np.all(decode.rms_norm(np.zeros((1, 5)), None, np.ones(5), 0.0, 1e-6)[1] == 0)


def test_scaled_groups_and_floor():
    v = np.array([[1.0, -2.0, 0.5, 8.0, 0.0]])
    grid, s = decode.scaled(v, 2, 127.0)
    np.testing.assert_allclose(s, [[2 / 127, 8 / 127, 2.0 ** -100 / 127]], rtol=1e-15)
    np.testing.assert_allclose(grid, [[63.5, -127.0, 0.5 / 8 * 127, 127.0, 0.0]], rtol=1e-15)
    grid, s = decode.scaled(v, 0, 448.0)
    assert s.shape == (1, 1) and s[0, 0] == pytest.approx(8 / 448)


def test_e4m3_format():
    vals = decode.e4m3_decode(np.arange(128))
    assert vals[0] == 0 and vals[1] == 2.0 ** -9 and vals[8] == 2.0 ** -6 and vals[0x38] == 1.0 and vals[126] == 448.0
    assert np.isnan(vals[127]) and np.all(np.diff(vals[:127]) > 0)
    assert np.array_equal(np.diff(vals[:127]), decode.e4m3_step(vals[:126]))
    assert decode.e4m3_decode(0x80 + 0x38) == -1.0


def test_nibble_order_and_weights():
    w = np.array([[0x21, 0x43, 0xF5]], dtype=np.uint8)
    assert decode.nibbles(w, 5).tolist() == [[1, 2, 3, 4, 5]]
    assert decode.nibbles(w, 6).tolist() == [[1, 2, 3, 4, 5, 15]]
    W = decode.w4_weights(np.full((1, 32), 0x98, np.uint8), np.array([[0.5, 2.0]]), np.array([[8, 0]], np.uint8), 64, 32)
    assert W[0, :4].tolist() == [0.0, 0.5, 0.0, 0.5] and W[0, 32:36].tolist() == [16.0, 18.0, 16.0, 18.0]
    assert np.array_equal(decode.w4_weights(np.full((1, 16), 0x08, np.uint8), np.ones((1, 1)), None, 32, 32)[0, :2],
                          [0.0, -8.0])


def test_attention_closed_forms():
    v = np.array([[1.0, 2.0], [3.0, 6.0]])
    o, lse = decode.attend(np.zeros(3), np.ones((2, 3)), v, 1.0)
    np.testing.assert_allclose(o, [2.0, 4.0])
    assert lse == pytest.approx(np.log(2))
    o, lse = decode.attend(np.array([np.log(3.0)]), np.array([[1.0], [0.0]]), v, 1.0)
    np.testing.assert_allclose(o, 0.75 * v[0] + 0.25 * v[1])
    assert lse == pytest.approx(np.log(4))
    o, lse = decode.attend(np.ones(2), np.zeros((0, 2)), np.zeros((0, 2)), 1.0)
    assert np.all(o == 0) and lse == -np.inf


@pytest.mark.parametrize("layout", ["head", "slot"])
def test_paged_attention_is_attention_over_the_gathered_rows(layout):
    rng = np.random.default_rng(1)
    kv, heads, dim, size = 2, 4, 8, 4
    k, v = rng.normal(size=(2, 6, kv, size, dim))
    if layout == "slot":
        ks, vs = k.transpose(0, 2, 1, 3).copy(), v.transpose(0, 2, 1, 3).copy()
    else:
        ks, vs = k, v
    q = rng.normal(size=(3, heads, dim))
    table = [[5, 0, 3], [2, 9, -1], [1, 1, 1]]          # page 9 does not exist: its positions are skipped
    out, lse = decode.paged_attention(q, ks, vs, table, [9, 6, 0], 0.3, layout=layout)
    rows = np.concatenate([k[5], k[0], k[3][:, :1]], 1), np.concatenate([v[5], v[0], v[3][:, :1]], 1)
    for h in range(heads):
        o, s = decode.attend(q[0, h], rows[0][h // 2], rows[1][h // 2], 0.3)
        np.testing.assert_allclose(out[0, h], o)
        assert lse[0, h] == pytest.approx(s)
        np.testing.assert_allclose(out[1, h], decode.attend(q[1, h], k[2, h // 2], v[2, h // 2], 0.3)[0])
    assert np.all(out[2] == 0) and np.all(np.isneginf(lse[2]))
    w, _ = decode.paged_attention(q, ks, vs, table, [9, 6, 0], 0.3, window=1, layout=layout)
    np.testing.assert_allclose(w[0], np.repeat(v[3][:, 0], 2, 0))
