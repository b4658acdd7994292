"""Pins of the key/value cache oracle: against the whole-state attention oracle, closed forms and hand-worked cases."""
import numpy as np

from oracle import bitrl_oracle as O
from oracle import cache_oracle as K
from paper_2604_24273_amd import synth


def _tables(n, dh, theta):
    inv = theta ** (-2.0 * np.arange(dh // 2) / dh)
    ang = np.arange(n)[:, None] * inv[None, :]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def _empty(pages, hkv, tokens, dh, states, table_pages, dtype=np.float32):
    row = (dh + 15) // 16 * 16
    c = {"k": np.zeros((pages, hkv, tokens, row), dtype), "v": np.zeros((pages, hkv, tokens, row), dtype),
         "table": np.arange(states * table_pages, dtype=np.int32).reshape(states, table_pages)[:, ::-1].copy()}
    if dtype == np.int8:
        c["k_scale"], c["v_scale"] = (np.zeros((pages, hkv, tokens), np.float32) for _ in range(2))
    return c


def test_tokens_one_by_one_equal_the_whole_state():
    hq, hkv, dh, n = 4, 2, 16, 11
    qkv = synth.normal(1, 1, (n, (hq + 2 * hkv) * dh))
    cos, sin = _tables(32, dh, 10000.0)
    want = O.causal_gqa_attention(qkv[:, :hq * dh].reshape(n, hq, dh), qkv[:, hq * dh:(hq + hkv) * dh].reshape(n, hkv, dh),
                                  qkv[:, (hq + hkv) * dh:].reshape(n, hkv, dh), 10000.0).reshape(n, -1)
    c = _empty(4, hkv, 4, dh, 1, 4)
    done = 0
    for step in (3, 1, 5, 2):
        rows = qkv[done:done + step]
        done += step
        K.append(c, rows, hq, None, [done], None, cos, sin)
        out, w, _ = K.attend(c, rows, hq, None, [done], None, cos, sin)
        assert np.abs(out - want[done - step:done]).max() < 3e-7
        assert np.allclose(w.sum(), step * hq)


def test_tree_of_one_branch_is_causal_and_siblings_do_not_see_each_other():
    hq, hkv, dh, n = 2, 1, 16, 4
    qkv = synth.normal(2, 1, (n, (hq + 2 * hkv) * dh))
    cos, sin = _tables(32, dh, 10000.0)
    c = _empty(2, hkv, 4, dh, 1, 2)
    K.append(c, qkv, hq, None, [n], None, cos, sin)
    chain = np.array([[1], [3], [7], [15]], dtype=np.uint32)
    a, _, reach = K.attend(c, qkv, hq, None, [n], None, cos, sin)
    b, _, _ = K.attend(c, qkv, hq, None, [n], None, cos, sin, chain)
    assert np.array_equal(a, b)
    assert np.all(reach >= np.abs(a).max(1)) and np.all(reach <= np.abs(qkv[:, (hq + hkv) * dh:]).max())
    alone = np.array([[1], [2], [4], [8]], dtype=np.uint32)       # each token sees itself only: its own value
    d, w, _ = K.attend(c, qkv, hq, None, [n], None, cos, sin, alone)
    v = qkv[:, (hq + hkv) * dh:]
    assert np.abs(d.reshape(n, hq, dh) - v[:, None]).max() < 1e-12 and np.allclose(w, hq)
    none, w, _ = K.attend(c, qkv, hq, None, [n], None, cos, sin, np.zeros((n, 1), np.uint32))
    assert np.array_equal(none, np.zeros_like(none)) and w.sum() == 0


def test_int8_rows_and_rotation_by_hand():
    codes, scale = K.quantise_row(np.array([0.0, 1.0, -2.0, 0.5], np.float32))
    assert codes.tolist() == [0, 64, -127, 32] and scale == np.float32(2) / np.float32(127)     # 63.5 and 31.75: ties to even
    codes, scale = K.quantise_row(np.zeros(4, np.float32))
    assert codes.tolist() == [0, 0, 0, 0] and scale > 0
    y = K.rotate(np.array([[1.0, 2.0, 3.0, 4.0]], np.float32), np.array([0.0, 1.0], np.float32), np.array([1.0, 0.0], np.float32))
    assert y.tolist() == [[-3.0, 2.0, 1.0, 4.0]]                  # pairs (1, 3) by 90 degrees, (2, 4) by 0


def test_select_and_compact_by_hand():
    w = np.array([[[9.0, 1.0, 5.0, 5.0, np.nan, 7.0, 0.0, 2.0]]], np.float32)
    kept, counts = K.select(w, [8], 5, 1, 1)
    assert kept.tolist() == [[[0, 2, 3, 5, 7]]] and counts.tolist() == [5]
    kept, counts = K.select(w, [8], 3, 1, 1)
    assert kept.tolist() == [[[0, 5, 7]]]
    kept, counts = K.select(w, [2], 3, 1, 1)
    assert kept.tolist() == [[[0, 1, -1]]] and counts.tolist() == [2]
    c = _empty(2, 1, 4, 16, 1, 2)
    c["k"][:] = np.arange(8).reshape(2, 1, 4, 1)[::-1]            # slot j holds j: the table counts pages backwards
    K.compact(c, [8], np.array([[[0, 5, 7]]]), None, [3], w)
    assert [c["k"][K.place(c, 0, j)[0], 0, K.place(c, 0, j)[1], 0] for j in range(8)] == [0, 5, 7, 3, 4, 5, 6, 7]
    assert w[0, 0, :3].tolist() == [9.0, 7.0, 2.0]
