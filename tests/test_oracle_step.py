"""Pins of the oracle of the step's operators: closed forms, other formulations, and the oracles that were there before."""
import numpy as np
import pytest

from oracle import step as O
from oracle import transformer as O2


def test_tables_hand_out_the_stack_from_its_top_in_request_order():
    table = np.full((3, 4), -1)
    table[0, 0], table[2, :2] = 7, (8, 9)
    start, kv, pos, slots, held, count, status, t = O.build_tables([14, 0, 33], [3, 0, 1], [1, 0, 2], [1, 2, 3, 4, 5], 4, table, 6)
    assert status == 0 and list(start) == [0, 3, 3, 4] and list(kv) == [17, 0, 34]
    assert list(pos) == [14, 15, 16, 33, -1, -1]
    assert list(t[0, :2]) == [7, 4] and list(t[2, :3]) == [8, 9, 3]           # entry 3 (value 4) is the top of a stack of four
    assert list(slots) == [7 * 16 + 14, 7 * 16 + 15, 4 * 16, 3 * 16 + 1, -1, -1]
    assert list(held) == [2, 0, 3] and count == 2


def test_held_blocks_behind_the_context_serve_the_next_step():
    table = np.array([[5, 6, -1]])
    _, _, pos, slots, held, count, status, t = O.build_tables([3], [14], [2], [9], 1, table, 14)
    assert status == 0 and held[0] == 2 and count == 1 and (t == table).all()
    assert slots[-1] == 6 * 16 and pos[-1] == 16


@pytest.mark.parametrize("ctx,new,held,count,rows,why", [([3], [-1], [1], 1, 9, -2), ([3], [40], [1], 9, 9, -8), ([3], [100], [1], 9, 999, -8),
                                                        ([3], [20], [1], 0, 99, -6), ([3], [20], [1], 10, 99, -2)])
def test_tables_hand_out_nothing_when_refused(ctx, new, held, count, rows, why):
    table = np.array([[4, -1, -1]])
    start, kv, pos, slots, h, c, status, t = O.build_tables(ctx, new, held, np.arange(9), count, table, rows)
    assert status == why and not start.any() and not kv.any() and (pos == -1).all() and (slots == -1).all()
    assert (t == table).all() and list(h) == held and c == count


def test_rotation_and_norm_agree_with_the_transformer_oracle():
    rng = np.random.default_rng(1)
    x, pos, g = rng.normal(size=(5, 3, 64)), np.array([0, 1, 77, 4000, 12]), rng.normal(1, 0.1, 64)
    y, _ = O.norm_rope(x, None, pos, 1e4, 1e-5)
    assert np.allclose(y, O2.rope(x, pos, 1e4), atol=1e-6)                     # (its tables are rounded to 32 bits)
    y, _ = O.norm_rope(x, g, np.zeros(5), 1e4, 1e-5)
    assert np.allclose(y, O2.rmsnorm(x, g, 1e-5), atol=1e-12)


def test_attention_without_a_window_is_the_transformer_oracles():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(4, 4, 64)), rng.normal(size=(9, 2, 64)), rng.normal(size=(9, 2, 64))
    want = O2.attention_rows(q, k, v, np.arange(5, 9), 2)
    for window, sinks in ((0, 0), (0, 3), (9, 0), (100, 2), (4, 5)):
        assert np.allclose(O.window_attention(q, k, v, 5, window, sinks)[0], want, atol=1e-12), (window, sinks)


def test_a_window_and_sinks_are_a_mask():
    assert list(O.visible(9, 3, 2)) == [0, 1, 7, 8, 9] and list(O.visible(1, 3, 4)) == [0, 1]
    assert list(O.visible(5, 1, 0)) == [5] and list(O.visible(-1, 4, 2)) == []


def test_verified_tokens_follow_the_target_whatever_the_draft():
    """The point of it: with drafts drawn from q, the first token is distributed as p (here with one draft and a fine grid of both random
    numbers, so that the frequencies are the probabilities up to the grid)."""
    p, q = np.array([0.5, 0.2, 0.25, 0.05]), np.array([0.1, 0.6, 0.05, 0.25])
    logits = np.log(np.stack([p, p]))
    n, got = 200, np.zeros(4)
    grid = (np.arange(n) + 0.5) / n
    for x in range(4):
        for u in grid:
            first = [int(O.verify_request(logits, [x], q[None], 1.0, [u], v)[0][0]) for v in (grid[::10] if u * q[x] >= p[x] else grid[:1])]
            for t in first:
                got[t] += q[x] / n / len(first)
    assert np.allclose(got, p, atol=0.03)


def test_verify_special_rows():
    V = 6
    z = np.zeros((3, V), np.float32)
    z[0, 2] = z[1, 4] = z[2, 1] = 5.0
    toks, a, _ = O.verify_request(z, [2, 4], None, 0.0, [0.9, 0.9], 0.3)
    assert list(toks) == [2, 4, 1] and a == 2
    toks, a, _ = O.verify_request(z, [2, 3], None, 0.0, [0.0, 0.0], 0.3)
    assert list(toks) == [2, 4, -1] and a == 1
    toks, a, _ = O.verify_request(np.full((2, V), np.nan), [3], None, 1.0, [0.0], 0.3)
    assert list(toks) == [0, -1] and a == 0
    # q covers p: drawn from p itself; a certain draft that is refused is never drawn
    p = np.full((2, V), 1 / V)
    toks, a, _ = O.verify_request(np.log(p), [1], p[:1] + 1e-3, 1.0, [0.9999], 0.0)
    assert a == 0 and list(toks) == [0, -1]
    toks, a, _ = O.verify_request(np.log(p), [0], None, 1.0, [0.5], 0.0)
    assert a == 0 and list(toks) == [1, -1]
    assert O.verify_request(np.log(p), [V], None, 1.0, [0.0], 0.999)[0][0] == V - 1
