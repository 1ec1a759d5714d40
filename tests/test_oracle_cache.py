"""The fp64 reference of the cache operators, against what fixes it."""
import numpy as np
import pytest

import oracle
import workloads as W
from oracle import cache as C


def bits(x):
    return W.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def test_every_value_of_the_format_is_its_own_code():
    for s in (0, 1, 100, 127, 200, 252):
        unit = 2.0 ** (s - 127)
        x = np.zeros((2, 32))
        x[0, :16] = np.concatenate([C.E2M1, -C.E2M1]) * unit
        x[0, 16:] = 6 * unit  # the largest element fixes the scale
        x[1] = 4 * unit
        codes, scales = C.kv4_quantise(bits(x))
        assert (scales[:, 0] == s).all()
        assert np.array_equal(C.kv4_values(codes, scales).reshape(2, 32), x)


def test_ties_go_to_the_even_code_and_large_elements_stop_at_six():
    x = np.zeros(32)
    x[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.5]
    got = C.kv4_values(*C.kv4_quantise(bits(x)))[0]
    assert np.array_equal(got[:8], [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0])


def test_quantisation_error_is_within_half_a_step():
    rng = np.random.default_rng(0)
    x = bits(rng.standard_normal((200, 64)) * np.exp(rng.uniform(-20, 20, (200, 1))))
    codes, scales = C.kv4_quantise(x)
    units = oracle.bf16_to_f64(x).reshape(200, 2, 32) / np.ldexp(1.0, scales.astype(int) - 127)[..., None]
    err = np.abs(C.kv4_values(codes, scales) / np.ldexp(1.0, scales.astype(int) - 127)[..., None] - units)
    m = np.abs(units)
    assert (m < 8).all() and (m.max(axis=-1) >= 4).all()
    half = np.where(m < 2, 0.25, np.where(m < 4, 0.5, np.where(m <= 6, 1.0, 2.0)))
    assert (err <= half).all()


def test_subnormal_zero_and_non_finite_groups():
    x = np.zeros((5, 32), dtype=np.uint16)
    x[1, 3] = 0x0001          # the smallest bf16
    x[2, 5], x[2, 6] = 0x7F80, 0x3F80  # an infinity
    x[3, 0] = 0xFFC0          # a NaN
    x[4, :] = 0x7F7F          # the largest finite bf16
    codes, scales = C.kv4_quantise(x)
    assert scales[:, 0].tolist() == [0, 0, 255, 255, 252]
    v = C.kv4_values(codes, scales)[:, 0]
    assert (v[0] == 0).all() and (v[1] == 0).all()
    assert np.isnan(v[2]).all() and np.isnan(v[3]).all()
    assert (v[4] == 6 * 2.0 ** 125).all()


def test_append_then_read_returns_the_quantised_rows():
    rng = np.random.default_rng(1)
    codes, scales = rng.integers(0, 256, (6, 2, 2, 16, 16), dtype=np.uint8), np.full((6, 2, 2, 16), 7, np.uint8)
    bt, lens = np.array([[3, 0], [5, 1]]), np.array([20, 3])
    new = bits(rng.standard_normal((2, 7, 2, 64)))
    c, s = C.kv4_append(codes, scales, new, bt, lens)
    back = C.kv4_read(c, s, 7, bt, lens)
    want = C.kv4_values(*C.kv4_quantise(new)).reshape(2, 7, 2, 64)
    assert np.array_equal(back[0], want[0])
    assert np.array_equal(back[1, 4:], want[1, 4:]) and (back[1, :4] == 0).all()
    touched = (c != codes).any(axis=-1) | (s != scales)
    where = np.argwhere(touched)
    assert {(n, t) for n, _, _, t in where.tolist()} <= {(3, 13), (3, 14), (3, 15), (0, 0), (0, 1), (0, 2), (0, 3), (5, 0),
                                                         (5, 1), (5, 2)}


@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 0), (9, 3), (9, 40), (1, 1)])
def test_visible_keys_against_the_masks(window, sinks):
    for length in (0, 1, 5, 40):
        for nq in (1, 3):
            for j in range(nq):
                p = length - nq + j
                want = [t for t in range(length) if t <= p and (window == 0 or p - t < window or t < sinks)]
                assert C.visible_keys(length, nq, j, window, sinks).tolist() == want


def test_attend_is_the_masked_oracle_without_sinks():
    w = W.build([1, 33, 100], 8, 2, 64, 16, seed=5, num_queries=2, window=20)
    got = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale,
                   window=20)
    ref = oracle.attend_masked(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, 20)[0]
    assert np.abs(got - ref).max() < 1e-12


def test_sinks_change_only_what_a_window_hides():
    w = W.build([100], 4, 2, 64, 16, seed=6, poison=False)
    k, v = oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache)
    args = (w.q[:, None], k, v, w.block_table, w.context_lens, w.scale)
    assert np.array_equal(C.attend(*args, window=30, sinks=70), C.attend(*args))  # 70 + 30 tokens: all of them
    far = C.attend(*args, window=30, sinks=4)
    assert np.abs(far - C.attend(*args, window=30)).max() > 1e-4
    assert np.array_equal(C.attend(*args, window=0, sinks=4), C.attend(*args))


# ---------------------------------------------------------------------- pages
def test_update_keeps_counts_tables_and_contents_together():
    """Random histories of a small cache whose tokens carry their sequence's own numbers: after every update, the
    copies and the appends, each row reads back what it should hold, and counts equal references."""
    page, n_pages, m = 4, 60, 8
    for seed in range(20):
        rng = np.random.default_rng(seed)
        pool = np.full((n_pages, page), -1)
        table, lens, count = np.full((1, m), -1, np.int32), np.zeros(1, np.int64), np.zeros(n_pages, np.int32)
        held = [[]]
        for _ in range(25):
            rows = int(rng.integers(1, 5))
            parents = rng.integers(-1, len(held), rows)
            new = np.array([max(0, min(m * page, (len(held[p]) if p >= 0 else 0) + int(rng.choice([-3, 0, 1, 1, 2, 6]))))
                            for p in parents])
            table, count, src, dst, info = C.pages_update(table, lens, parents, new, count, page)
            assert info[1] == 0
            before = pool.copy()
            for a, b in zip(src, dst):
                if b >= 0:
                    pool[b] = before[a]
            kept = [held[p][:n] if p >= 0 else [] for p, n in zip(parents, new)]
            held = [k + rng.integers(0, 1000, n - len(k)).tolist() for k, n in zip(kept, new)]
            for r, (k, h) in enumerate(zip(kept, held)):
                for t in range(len(k), len(h)):
                    pool[table[r, t // page], t % page] = h[t]
            lens = new
            for r, h in enumerate(held):
                assert [pool[table[r, t // page], t % page] for t in range(len(h))] == h
                assert (table[r, -(-len(h) // page):] == -1).all()
            used = table[table >= 0]
            assert np.array_equal(np.bincount(used, minlength=n_pages), count)
            table2, count2, page_map, s2, d2, info2 = C.pages_compact(table, lens, count, page)
            before = pool.copy()
            pool[d2[:info2[1]]] = before[s2[:info2[1]]]
            assert (count2[:info2[0]] > 0).all() and (count2[info2[0]:] == 0).all()
            table, count = table2, count2
            for r, h in enumerate(held):
                assert [pool[table[r, t // page], t % page] for t in range(len(h))] == h


def test_update_releases_what_a_window_hides_and_keeps_sinks():
    page, table = 4, np.arange(10, dtype=np.int32)[None]
    out, count, *_ = C.pages_update(table, [40], None, [41], np.ones(12, np.int32), page, window=9, sinks=5)
    assert out.shape == (1, 10)  # 41 tokens are clamped to the table's 40
    assert out[0].tolist() == [0, 1, -1, -1, -1, -1, -1, 7, 8, 9]
    assert count.tolist() == [1, 1, 0, 0, 0, 0, 0, 1, 1, 1, 1, 1]
