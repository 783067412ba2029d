"""The oracle of the decoder block's pieces against hand-worked numbers, closed forms and library routines (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD


def test_e4m3_codes_against_the_library_cast_and_by_hand():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 9, 4000), [0.0, -0.0, 448.0, 447.9, -448.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.01, 0.01]])
    want = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(OD.e4m3_encode(x.astype(np.float32)), want)
    assert list(OD.e4m3_encode([1.0, 1.0625, 1.1875, 500.0, -1e9, np.nan])) == [0x38, 0x38, 0x3A, 0x7E, 0xFE, 0x7F]      # ties to the even code, saturation
    codes = np.arange(256, dtype=np.uint8)
    codes = codes[(codes & 0x7F) != 0x7F]
    assert np.array_equal(OD.e4m3_encode(OD.e4m3_decode(codes)), codes)


def test_rms_norm_hand_worked_row_and_scale_invariance():
    s, y = OD.add_rms_norm(np.array([[3.0, 1.0]]), np.array([[0.0, 3.0]]), np.array([2.0, 1.0]), 0.0)
    assert np.allclose(s, [[3.0, 4.0]]) and np.allclose(y, [[6.0 / np.sqrt(12.5), 4.0 / np.sqrt(12.5)]])
    x = np.random.default_rng(2).standard_normal((5, 64))
    assert np.allclose(OD.add_rms_norm(x, None, np.ones(64), 0.0)[1], OD.add_rms_norm(7.0 * x, None, np.ones(64), 0.0)[1])
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), eps=1e-3).numpy()
    assert np.allclose(OD.add_rms_norm(x, None, np.ones(64), 1e-3)[1], want)


def test_rotary_keeps_lengths_and_scores_depend_on_distance_alone():
    rng = np.random.default_rng(3)
    table, x, y = OD.rotary_table(40, 64), rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    at = lambda v, p: OD.rotate(v, table, np.array([[p, p, p]]), (32, 0, 0))
    assert np.allclose(np.linalg.norm(at(x, 17)), np.linalg.norm(x)) and np.allclose(at(x, 0), x)
    assert np.allclose((at(x, 20) * at(y, 13)).sum(), (at(x, 9) * at(y, 2)).sum())
    # a quarter turn of pair 0 alone: the pair's partner lies half a head away
    table[:, :, 0], table[:, :, 1] = 1.0, 0.0
    table[5, 0] = (0.0, 1.0)
    e = np.zeros((1, 1, 64))
    e[0, 0, 0] = 1.0
    assert at(e, 5)[0, 0, 32] == 1.0 and at(e, 5)[0, 0, 0] == 0.0
    # three axes: each pair follows its own
    t = OD.rotary_table(40, 64)
    got = OD.rotate(x, t, np.array([[3, 11, 29]]), (20, 8, 4))
    for pairs, p in (((0, 20), 3), ((20, 28), 11), ((28, 32), 29)):
        one = OD.rotate(x, t, np.array([[p, p, p]]), (32, 0, 0))
        for i in (0, 32):
            assert np.allclose(got[..., i + pairs[0]: i + pairs[1]], one[..., i + pairs[0]: i + pairs[1]])


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -96), (3e38, 120)])
def test_block_exponents_by_hand(amax, e):
    assert OD.block_exponent(amax) == e


@pytest.mark.parametrize("steps", [[70], [1] * 70, [31, 1, 1, 37], [32, 32, 6], [5, 60, 5]])
def test_a_cache_filled_in_steps_holds_the_tokens(steps):
    """Whatever the steps: every value within a code's rounding under the block's final scale (and a second one where it grew), the same scales."""
    rng = np.random.default_rng(4)
    K, V = (rng.standard_normal((70, 2, 64)) * np.exp(rng.standard_normal((70, 1, 1))) for _ in range(2))
    c, pages, at = OD.Cache(4, 2, 64, rng), [3, 1], 0
    for n in steps:
        c.append(pages, at, K[at: at + n], V[at: at + n])
        at += n
    whole = OD.Cache(4, 2, 64)
    whole.append(pages, 0, K, V)
    for block in range(3):
        p, half = pages[block // 2], block % 2
        assert np.array_equal(c.scales[p, :, :, half], whole.scales[p, :, :, half])
    for X, got, which in ((K, c.values(pages, 70)[0], 0), (V, c.values(pages, 70)[1], 1)):
        step = 2.0 ** (np.array([c.scales[pages[t // 64], :, which, t % 64 // 32] for t in range(70)]).astype(float) - 127)[:, :, None]
        bound = np.maximum(np.abs(X) * 2.0 ** -4, step * 2.0 ** -10)
        assert (np.abs(got - X) <= bound * 1.0001 + step * 2.0 ** -10).all()


def test_padding_joins_nothing_and_a_nan_is_held_in_the_key():
    c = OD.Cache(1, 1, 64)
    K, V = np.ones((5, 1, 64)), np.ones((5, 1, 64))
    V[3, 0, 7] = np.nan
    K[4, 0, 9] = np.inf
    c.append([0], -2, K, V)
    k, v = c.values([0], 3)
    assert np.isnan(k[1, 0, 0]) and v[1, 0, 7] == 0.0 and (k[0] == 1.0).all() and not np.isnan(v).any()
    assert k[2, 0, 9] == 448.0 * 2.0 ** -8 and k[2, 0, 8] == 1.0             # an infinity is the largest code and does not move the scale
    assert (c.codes[0, 0, :, 3:] == 0).all()


def test_packed_order_is_a_permutation_that_the_chunk_formulas_name():
    c = OD.Cache(1, 1, 128)
    c.codes[:] = np.random.default_rng(5).integers(0, 256, c.codes.shape)
    p = c.packed()[0, 0]
    assert sorted(p[0]) == sorted(c.codes[0, 0, 0].reshape(-1))
    for t, ch in ((0, 0), (5, 3), (37, 7), (63, 1)):
        at = ((((t // 4) % 4) * 8 + ch) * 16 + 4 * (t // 16) + t % 4) * 16
        assert np.array_equal(p[0, at: at + 16], c.codes[0, 0, 0, t, 16 * ch: 16 * ch + 16])
    for d, q in ((0, 0), (17, 2), (127, 3)):
        at = (((d // 16) * 4 + q) * 16 + d % 16) * 16
        assert np.array_equal(p[1, at: at + 16], c.codes[0, 0, 1, 16 * q: 16 * q + 16, d])


@pytest.mark.parametrize("window,softcap", [(0, 0.0), (3, 0.0), (0, 5.0), (1, 2.0)])
def test_attention_against_the_library_routine(window, softcap):
    rng = np.random.default_rng(6)
    Q, K, V = rng.standard_normal((4, 6, 64)), rng.standard_normal((9, 3, 64)), rng.standard_normal((9, 3, 64))
    o, _ = OD.attention(Q, K, V, 5, 0.125, window, softcap)
    k, v = (torch.from_numpy(x).repeat_interleave(2, 1).permute(1, 0, 2) for x in (K, V))
    z = torch.from_numpy(Q).permute(1, 0, 2) @ k.transpose(1, 2) * 0.125
    if softcap:
        z = softcap * torch.tanh(z / softcap)
    i, j = torch.arange(5, 9)[:, None], torch.arange(9)[None]
    z = z.masked_fill((j > i) | ((j <= i - window) if window else (j < 0)), -np.inf)
    assert np.allclose(o, (torch.softmax(z, 2) @ v).permute(1, 0, 2).numpy())


def test_rows_that_see_nothing_are_zeros_and_nans_reach_only_who_sees_them():
    rng = np.random.default_rng(7)
    Q, K, V = rng.standard_normal((4, 1, 64)), rng.standard_normal((2, 1, 64)), rng.standard_normal((2, 1, 64))
    K[1, 0, 0] = np.nan
    o, _ = OD.attention(Q, K, V, -2, 1.0)
    assert (o[:2] == 0).all() and np.allclose(o[2, 0], V[0, 0]) and np.isnan(o[3]).all()


def test_pages_fork_free_and_compact_by_hand():
    p = OD.Pages(8)
    a = p.take(3)
    assert a == [0, 1, 2]
    child, moves = p.fork(a, 130)                                # two whole pages and two tokens of a third
    assert child == [0, 1, 3] and moves == [(2, 3)] and p.refs[:4] == [2, 2, 1, 1]
    p.free(a)
    assert p.refs[:4] == [1, 1, 0, 1] and p.free_pages[-1] == 2
    moves, tables = p.compact([child])
    assert moves == [(3, 2)] and tables == [[0, 1, 2]] and p.free_pages == [7, 6, 5, 4, 3]
    assert p.fork([0, 1, 2], 128) == ([0, 1], [])
