"""Pins of the operator oracle on cases worked out by hand, and the host-only halves of the calls (no GPU)."""
import numpy as np
import pytest

from oracle import operators as oo
from paper_2411_09317_b200 import binding as pie


def test_rotation_is_a_turn_of_each_pair_by_its_axis():
    x = np.zeros((2, 1, 8))
    x[0, 0] = [1, 0, 2, 0, 0, 0, 0, 3]
    # halves: pairs (0, 4), (1, 5) of rotary_dim 4 ... here rotary 8: (0, 4), (1, 5), (2, 6), (3, 7)
    axis, freq = [0, 0, 1, 1], [np.pi / 2, 1.0, np.pi, np.pi / 2]
    y, size = oo.rotate(x, np.array([[1, 0], [1, 0]]), axis, freq)
    assert np.allclose(y[0, 0], [0, 0, -2, -3, 1, 0, 0, 0], atol=1e-15)
    assert np.allclose(y[1], x[1])
    assert np.allclose(size[0, 0], [1, 0, 2, 3, 1, 0, 2, 3])
    y, _ = oo.rotate(x, np.array([[1, 0], [1, 0]]), axis, freq, adjacent=True, amplitude=2.0)
    assert np.allclose(y[0, 0], [0, 2, 4 * np.cos(1), 4 * np.sin(1), 0, 0, -6, 0], atol=1e-15)


def test_rotation_depends_on_position_differences_only():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    freq = 10000.0 ** (-np.arange(32) / 32)
    dots = []
    for base in (0, 12345, 1 << 30):
        a, _ = oo.rotate(q, np.array([[base + 7]]), [0] * 32, freq)
        b, _ = oo.rotate(k, np.array([[base]]), [0] * 32, freq)
        dots.append(float((a * b).sum()))
    assert np.allclose(dots, dots[0], atol=1e-9)


def test_prompt_attention_by_hand():
    q = np.zeros((3, 2, 2))
    k = np.ones((3, 1, 2))
    v = np.arange(6.0).reshape(3, 1, 2)
    out, size = oo.prompt_attention(q, k, v, [0, 1, 3], 1.0)      # zero queries: plain means over what is seen
    assert np.allclose(out[0], [[0, 1]] * 2) and np.allclose(out[1], [[2, 3]] * 2) and np.allclose(out[2], [[3, 4]] * 2)
    assert np.allclose(size, out)


def test_weights_of_a_group_add_up_to_its_heads():
    rng = np.random.default_rng(1)
    w = oo.attention_weights(rng.standard_normal((6, 16)), rng.standard_normal((11, 2, 16)), 0.25)
    assert w.shape == (2, 11) and np.allclose(w.sum(1), 3.0)
    assert oo.attention_weights(np.zeros((2, 4)), np.zeros((0, 1, 4)), 1.0).shape == (1, 0)


def test_kept_positions_by_hand():
    w = [5, 1, 5, 5, 9, 0, 0]
    assert oo.keep(w, 7, 7, 2) == list(range(7))
    assert oo.keep(w, 7, 4, 2) == [0, 4, 5, 6]          # 9, then the first of the fives, then the newest two
    assert oo.keep(w, 7, 3, 3) == [4, 5, 6]
    assert oo.keep(w, 7, 3, 0) == [0, 2, 4]
    assert oo.keep([np.nan, -1.0, -2.0, 0.0], 4, 2, 0) == [1, 3]
    assert oo.keep([], 0, 1, 1) == []


@pytest.mark.parametrize("pos", [1, 4097, 1_000_003, (1 << 31) - 1, -5, -(1 << 31)])
def test_fixed_point_angles_keep_their_fraction(pos):
    """The low word of position * turns is the angle's fraction of a turn: 2^-33 of a turn in the frequency, times 2^31
    positions, plus the extended-precision product it is held against."""
    freq = 500000.0 ** (-np.arange(0, 128, 2) / 128.0)
    turns, n_axes = pie.pie_rope_plan(128, 128, np.arange(64) % 3, freq)
    assert n_axes == 3
    two_pi = 2 * np.longdouble("3.14159265358979323846264338327950288")
    for i in range(64):
        got = ((pos * int(turns[i])) % (1 << 64)) / 2.0 ** 64
        want = np.longdouble(pos) * np.longdouble(freq[i]) / two_pi
        diff = float((want - np.floor(want)) - np.longdouble(got))
        assert min(abs(diff), 1 - abs(diff)) < 2.0 ** -30, (i, diff)


def test_frequencies_of_whole_and_negative_turns():
    turns, n_axes = pie.pie_rope_plan(64, 16, [0] * 8, [0.0, 2 * np.pi, -np.pi / 2, np.pi / 2, 7 * np.pi, 1e-30, -1e-30, 1e6])
    assert n_axes == 1 and turns[0] == 0
    assert min(int(turns[1]), (1 << 64) - int(turns[1])) < 1 << 14        # 2 pi in double is a whole turn to 2^-52
    assert abs(int(turns[2]) - (3 << 62)) < 1 << 14 and abs(int(turns[3]) - (1 << 62)) < 1 << 14
    assert int(turns[5]) == 0 and int(turns[6]) == 0


@pytest.mark.parametrize("args,status", [
    ((128, 0, [0], [1.0]), pie.PIE_ERR_INVALID), ((64, 80, [0] * 40, [1.0] * 40), pie.PIE_ERR_INVALID),
    ((128, 24, [0] * 12, [1.0] * 12), pie.PIE_ERR_UNSUPPORTED), ((128, 16, [0] * 7 + [4], [1.0] * 8), pie.PIE_ERR_INVALID),
    ((128, 16, [0] * 7 + [-1], [1.0] * 8), pie.PIE_ERR_INVALID), ((128, 16, [0] * 8, [1.0] * 7 + [np.inf]), pie.PIE_ERR_INVALID),
    ((128, 16, [0] * 8, [np.nan] + [1.0] * 7), pie.PIE_ERR_INVALID)])
def test_rope_plan_refuses(args, status):
    with pytest.raises(pie.PieError) as e:
        pie.pie_rope_plan(*args)
    assert e.value.status == status


@pytest.mark.parametrize("lens", [[1], [0, 0], [64, 65, 0, 1, 1000, 64], [5] * 40, [100000, 3]])
@pytest.mark.parametrize("item", [64, 256, 84])
def test_prompt_plan_covers_every_token_once_longest_first(lens, item):
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    items = pie.pie_prompt_plan(off, item)
    seen = np.zeros(int(off[-1]), np.int32)
    for first, tok, n, s in items:
        assert first == off[s] and n == lens[s] and tok % item == 0 and tok < n
        seen[first + tok:first + min(tok + item, n)] += 1
    assert np.all(seen == 1)
    assert np.all(np.diff(items[:, 1]) <= 0)          # an item sees the keys up to its last token: the longest first


@pytest.mark.parametrize("off", [[1, 2], [0, 5, 4], [0, -1]])
def test_prompt_plan_refuses(off):
    with pytest.raises(pie.PieError) as e:
        pie.pie_prompt_plan(off, 64)
    assert e.value.status == pie.PIE_ERR_INVALID
    with pytest.raises(pie.PieError):
        pie.pie_prompt_plan([0, 5], 0)


def test_calls_without_a_pool_are_refused():
    i, u = pie.PIE_ERR_INVALID, np.zeros(4, np.int32)
    for call in (lambda: pie.pie_set_rope(None, 16, [0] * 8, [1.0] * 8),
                 lambda: pie.pie_rope_kv_write(None, 0, 16, 16, 16, 16, 16, 16, 16, 16, 1, 16, 1, 1),
                 lambda: pie.pie_prompt_attention(None, 16, 16, 16, 32, u, 1, 1.0),
                 lambda: pie.pie_decode_attention_weights(None, 0, 16, 16, 16, 1, 16, 1, 1.0, 16, 1),
                 lambda: pie.pie_kv_evict(None, 0, 16, 1, 16, 1, 16, 1, 1, 0)):
        with pytest.raises(pie.PieError) as e:
            call()
        assert e.value.status == i
