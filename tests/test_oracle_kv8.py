"""The 8-bit cache's oracle against hand-worked cases and closed forms (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K


def test_codes_are_torchs():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    np.testing.assert_array_equal(codes.view(torch.float8_e4m3fn).float().numpy().astype(np.float64), K.CODES)
    x = np.concatenate([np.linspace(-448, 448, 40001), np.linspace(-0.05, 0.05, 20001)])
    ref = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert K.same_codes(K.encode(x.astype(np.float32)), ref)


@pytest.mark.parametrize("a,c,s", [(448.0, 448, 1.0), (448.0001, 448, 2.0), (224.0, 448, 0.5), (1.0, 448, 2.0 ** -8), (0.875, 448, 2.0 ** -9),
                                   (0.0, 448, 2.0 ** -100), (1e-38, 448, 2.0 ** -100), (127.0, 127, 1.0), (127.5, 127, 2.0), (63.5, 127, 0.5)])
def test_power_of_two_scale(a, c, s):
    assert K.pow2(a, float(c)) == s


def test_page_by_hand():
    """One head of four dimensions: a page of two tokens, then a larger one that moves its scale."""
    p = K.new_pool(1, 1, 1, 4)
    x = np.array([[1.0, -2.0, 3.0, 0.0], [0.5, 0.5, -7.0, 0.01]])
    K.append(p, x[None, None, :, None], x[None, None, :, None], [[0]], [0], [2])
    assert p["scale"][0, 0, 0].tolist() == [2.0 ** -6, 2.0 ** -6]              # 7 * 64 = 448
    np.testing.assert_array_equal(K.CODES[p["k"][0, 0, 0, :2]], [[64, -128, 192, 0], [32, 32, -448, 0.625]])
    np.testing.assert_array_equal(p["v"][0, 0, 0, :, :2].T, p["k"][0, 0, 0, :2])
    # sums 96, -96, -256, 0.625 over 4: 256 / 4 = 64 <= 127 < 256 / 2
    assert p["summary"][0, 0, 0].tolist() == [24, -24, -64, 0] and p["summary_scale"][0, 0, 0] == 4 * 2.0 ** -6
    y = np.array([[0.0, 0.0, 0.0, 700.0]])
    K.append(p, y[None, None, :, None], y[None, None, :, None], [[0]], [2], [1])
    assert p["scale"][0, 0, 0, 0] == 2.0                                        # 700 <= 448 * 2
    # 1 / 2, 2 / 2, 3 / 2; 0.625 / 128 = 2.5 steps of 2^-9, a tie, to the even code 2
    np.testing.assert_array_equal(K.CODES[p["k"][0, 0, 0, :3]], [[0.5, -1, 1.5, 0], [0.25, 0.25, -3.5, 2 * 2.0 ** -9], [0, 0, 0, 352]])


def test_rotation_is_the_angle():
    ang = np.array([[0.3, 1.1]])
    x = np.array([1.0, 2.0, 3.0, 4.0, 5.0])
    y = K.rotate(x, 0, np.cos(ang), np.sin(ang), False)
    z = np.array([1 + 3j, 2 + 4j]) * np.exp(1j * ang[0])
    np.testing.assert_allclose(y, [z[0].real, z[1].real, z[0].imag, z[1].imag, 5.0])
    y = K.rotate(x, 0, np.cos(ang), np.sin(ang), True)
    z = np.array([1 + 2j, 3 + 4j]) * np.exp(1j * ang[0])
    np.testing.assert_allclose(y, [z[0].real, z[0].imag, z[1].real, z[1].imag, 5.0])


def _random_pool(rng, pages, H, D, ctx):
    p = K.new_pool(1, pages, H, D)
    B = len(ctx)
    per = pages // B
    table = rng.permutation(pages).reshape(B, per)
    for b in range(B):
        x, y = rng.standard_normal((2, 1, 1, ctx[b], H, D))
        one = lambda a: a  # noqa: E731
        K.append(p, one(x), y, [table[b]], [0], [ctx[b]])
    return p, table


def test_attention_by_brute_force_and_selection_of_all_pages():
    rng = np.random.default_rng(3)
    ctx = [37, 0, 16]
    p, table = _random_pool(rng, 9, 2, 8, ctx)
    q = rng.standard_normal((3, 3, 4, 8))
    kb, vb = rng.standard_normal((2, 3, 3, 2, 8))
    out, mag = K.attention(q, kb, vb, p, 0, table, ctx)
    for b in range(3):
        for j in range(3):
            for hq in range(4):
                w, acc, top = 0.0, np.zeros(8), np.zeros(8)
                for t in range(ctx[b] + j + 1):
                    if t < ctx[b]:
                        ph, s = table[b][t // 16], p["scale"][0, table[b][t // 16], hq // 2]
                        k, v = K.CODES[p["k"][0, ph, hq // 2, t % 16]] * s[0], K.CODES[p["v"][0, ph, hq // 2, :, t % 16]] * s[1]
                    else:
                        k, v = kb[b, t - ctx[b], hq // 2], vb[b, t - ctx[b], hq // 2]
                    e = math.exp(float(q[b, j, hq] @ k) / math.sqrt(8))
                    w, acc, top = w + e, acc + e * v, top + e * np.abs(v)
                np.testing.assert_allclose(out[b, j, hq], acc / w, atol=1e-12)
                np.testing.assert_allclose(mag[b, j, hq], top / w, atol=1e-12)
    sel = K.select(q, p, 0, table, ctx, 3, 1, 1)
    assert sel[0, 0, 0].tolist() == [0, 1, 2] and sel[1, 0, 0].tolist() == [-1] * 3 and sel[2, 2, 1].tolist() == [0, -1, -1]
    np.testing.assert_array_equal(K.attention(q, kb, vb, p, 0, table, ctx, sel=sel)[0], out)
    # the full mask sees every block row from every row
    full = K.attention(q, kb, vb, p, 0, table, ctx, full=True)[0]
    np.testing.assert_allclose(full[:, 2], out[:, 2])
    assert not np.allclose(full[:, 0], out[:, 0])


def test_selection_by_hand():
    """Eight pages whose summaries are multiples of one direction: the scores are those multiples."""
    p = K.new_pool(1, 8, 1, 4)
    for i, w in enumerate((5, 9, 9, -3, 9, 7, 0, 1)):
        p["summary"][0, i, 0] = (w, 0, 0, 0)
        p["summary_scale"][0, i, 0] = 0.5
    q = np.zeros((1, 1, 2, 4))
    q[0, 0, 0, 0], q[0, 0, 1, 0] = 1.0, -1.0
    table = np.arange(8)[None]
    pick = lambda n, s, r: K.select(q[:, :, :1], p, 0, table, [128], n, s, r)[0, 0, 0].tolist()  # noqa: E731
    assert pick(3, 0, 0) == [1, 2, 4]
    assert pick(2, 0, 0) == [1, 2]                # a tie of three goes to the lower pages
    assert pick(4, 1, 2) == [0, 1, 6, 7]
    assert pick(3, 1, 2) == [0, 6, 7]
    # the larger of the two heads' products: page 3 scores |-3|
    assert K.select(q, p, 0, table, [128], 6, 0, 0)[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5]
