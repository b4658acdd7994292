"""GPU tests of what numbers the key/value cache and its attention carry: rows of very different size side by side, long flat tails
behind one dominant key, new rows that are no numbers.

Bounds.  Every (token, head) is judged by its own sum_j p_j |v_j| over the slots that it sees (the largest of its components), never
by another's.  As in the other cache tests 2e-6 of that for scores of unit scale, and on top what the operands' two fp16 planes do not
hold: a half step of the smallest fp16 number is 2^-25, and a row's largest probability is carried as 2^12 at least, so each probability is off by
at most 2^-37 of the largest, the output by 2^-37 sum_j |v_j|.  (int8: products of probability and scale, the largest as 2^10 at least, so
each is off by 2^-35 of the largest, which is a share of the bound below 1e-7 for the few thousand slots here.)
Values of an fp32 cache are such pairs themselves, taken as they are: off by at most 2^-25 each, and so is their average.
"""
import numpy as np
import pytest

from oracle import cache_oracle as K
from paper_2604_24273_amd import synth
from test_gpu_cache import DTYPES, OnGpu, REL, _mods, ancestors, make_cache, same_bits, tables

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def by_head(c, qkv, hq, hkv, dh, cu, lens, positions, cos, sin, tree):
    """The oracle one query head at a time: out [T, hq, dh], reach [T, hq]."""
    T, group = qkv.shape[0], hq // hkv
    rows = qkv.reshape(T, hq + 2 * hkv, dh)
    outs, reaches = [], []
    for h in range(hq):
        g = h // group
        one = {n: x if n == "table" else x[:, g:g + 1] for n, x in c.items()}
        out, _, reach = K.attend(one, np.ascontiguousarray(rows[:, [h, hq + g, hq + hkv + g]]).reshape(T, -1), 1, cu, lens, positions, cos, sin, tree)
        outs.append(out)
        reaches.append(reach)
    return np.stack(outs, 1), np.stack(reaches, 1)


def check_each(got, want, bound):
    """got [T, hq * dh], want [T, hq, dh], bound [T, hq]"""
    diff = np.abs(got.reshape(want.shape).astype(np.float64) - want).max(-1)
    part = diff / bound
    at = np.unravel_index(np.nanargmax(part), part.shape)
    print("   worst %.3f of the bound %.1e at token %d, head %d" % (part[at], bound[at], *at), flush=True)
    assert np.all(np.isfinite(got)) and np.all(diff <= bound), (at, diff[at], bound[at])


def setting(dh, hq, hkv, page, cached, new, mask, dtype, seed):
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rng = np.random.default_rng(seed + dh + sum(cached))
    qkv = synth.normal(seed, dh + int(cu[-1]), (int(cu[-1]), (hq + 2 * hkv) * dh))
    cos, sin = tables(max(lens), dh)
    c = make_cache(seed + 1, hkv, dh, page, lens, DTYPES[dtype])
    words = -(-max(new) // 32)
    tree = None if mask == "causal" else np.concatenate([ancestors(rng, n, words) for n in new])
    return lens, cu, rng, qkv, cos, sin, c, tree


SIZES = [
    # (head_dim, heads, kv heads, page, cached, new)
    (128, 4, 4, 16, [40, 0, 3], [9, 5, 16]),                      # a workgroup each
    (16, 8, 2, 16, [20], [4]),
    (128, 20, 5, 32, [1700, 31], [3, 2]),                         # the shared list
    (32, 8, 8, 64, [100, 31], [33, 2]),                           # keys shared by many rows
    (100, 3, 3, 32, [900], [50]),                                 # and split
    (64, 4, 2, 32, [100, 0], [40, 20]),                           # two row tiles per wavefront
    (128, 8, 2, 64, [10, 0], [130, 33]),
]


# ---------------------------------------------------------------- rows of very different size

@pytest.mark.parametrize("ratio", [2.0 ** 10, 2.0 ** 31, 2.0 ** 60])
@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", SIZES)
def test_large_int8_rows_stay_with_the_tokens_that_see_them(dh, hq, hkv, page, cached, new, mask, ratio):
    """New tokens whose value rows are far larger than all others: who does not see them is as exact as without them."""
    B, R = _mods()
    print("large rows", dh, hq, hkv, page, cached, new, mask, ratio, flush=True)
    lens, cu, _, qkv, cos, sin, c, tree = setting(dh, hq, hkv, page, cached, new, mask, "i8", 61)
    for b, n in enumerate(new):
        for i in {n // 2, n - 1}:
            slot = cached[b] + i
            c["v_scale"][c["table"][b, slot // page], :, slot % page] *= np.float32(ratio)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, tree=tree)
    want, reach = by_head(c, qkv, hq, hkv, dh, cu, lens, None, cos, sin, tree)
    check_each(got, want, REL * reach)                            # (2^-37 of a few hundred rows: nothing)


@pytest.mark.parametrize("new", [1, 33])
@pytest.mark.parametrize("cached", [100, 3000])
@pytest.mark.parametrize("slot", [0, 50])
def test_large_int8_rows_of_no_weight(slot, cached, new):
    """A value row 2^31 times the others that every token sees, under a key whose probability is 2^-100 and less: in front of the
    other keys and between them."""
    B, R = _mods()
    dh, page = 64, 32
    lens = [cached + new]
    cos, sin = tables(lens[0], dh)
    c = make_cache(63, 1, dh, page, lens, np.int8)
    qkv = synth.normal(63, new, (new, 3 * dh))
    qkv[:, :dh] = 1.0                                             # at position 0: no rotation
    pg, at = c["table"][0, slot // page], slot % page
    c["k"][pg, 0, at, :dh], c["k_scale"][pg, 0, at] = -127, 12.0 / 127          # score -12 * 64 / 8 = -96, in bits -138
    c["v_scale"][pg, 0, at] *= np.float32(2.0 ** 31)
    positions = np.zeros(new, np.int32)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, 1, None, new, lens, positions=positions)
    want, reach = by_head(c, qkv, 1, 1, dh, None, lens, positions, cos, sin, None)
    check_each(got, want, REL * reach)


@pytest.mark.parametrize("size", [1e-24, 1e-12, 1.0, 1e4])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", SIZES)
def test_weights_do_not_follow_the_size_of_int8_values(dh, hq, hkv, page, cached, new, size):
    """Value rows of any size, and some of zeros between them: the softmax weights are those of the scores."""
    B, R = _mods()
    lens, cu, rng, qkv, cos, sin, c, _ = setting(dh, hq, hkv, page, cached, new, "causal", "i8", 71)
    c["v_scale"] *= np.float32(size)
    c["v_scale"] = np.where(rng.random(c["v_scale"].shape) < 0.1, np.float32(1e-30) / np.float32(127), c["v_scale"])
    w = torch.zeros(len(lens), hkv, max(lens), device="cuda")
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, weights=w)
    want, added, _ = K.attend(c, qkv, hq, cu, lens, None, cos, sin)
    g = w.cpu().numpy()
    assert np.all(np.abs(g - added) <= 4e-6 * added + 2.0 ** -23 * g)
    want, reach = by_head(c, qkv, hq, hkv, dh, cu, lens, None, cos, sin, None)
    # values below 1e-23: products with a scale of 2^-86 are carried as 2^(10 + 75 - 86) = 1/2 at least, to 2^-25.  Scales below 2^-75 count
    # as that, so a token that sees nothing but rows of a scale of 2^-107 (state 2's first token is one, with such a row of codes up to 127) has
    # its sum of probabilities carried as 2^(10 + 75) at least, each product to 2^-25, codes to 127: off by 127 * 2^-25 * 2^-85 at most.
    check_each(got, want, (REL + (2.0 ** -23 if size < 1e-20 else 0.0)) * reach + 127 * 2.0 ** -110)


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", SIZES)
def test_value_rows_of_different_size(dh, hq, hkv, page, cached, new, mask, dtype):
    """Value rows from 1e-3 to 1e4: the large ones are new tokens that some others do not see."""
    B, R = _mods()
    print("sizes", dh, hq, hkv, page, cached, new, mask, dtype, flush=True)
    lens, cu, rng, qkv, cos, sin, c, tree = setting(dh, hq, hkv, page, cached, new, mask, dtype, 65)
    for b, n in enumerate(new):
        size = np.concatenate([10.0 ** rng.uniform(-3, 0, cached[b]), 10.0 ** rng.uniform(-3, 4, n)])
        for slot, x in enumerate(size):
            pg, at = c["table"][b, slot // page], slot % page
            name = "v_scale" if dtype == "i8" else "v"
            c[name][pg, :, at] = (c[name][pg, :, at].astype(np.float64) * x).astype(c[name].dtype)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, tree=tree)
    want, reach = by_head(c, qkv, hq, hkv, dh, cu, lens, None, cos, sin, tree)
    # (scores of unit scale lie within 15 bits, so that 2^-37 of the largest probability is 2^-22 of any)
    check_each(got, want, REL * reach + (2.0 ** -25 if dtype == "f32" else 0.0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("new", [1, 20, 80])
@pytest.mark.parametrize("first", [True, False])
def test_a_long_flat_tail_behind_one_key(first, new, dtype):
    """One key 20 bits above 60000 equal ones, its value row zero: the output is the tail's, whose probabilities are about 2^-20 each."""
    B, R = _mods()
    print("tail", first, new, dtype, flush=True)
    dh, page, cached = 64, 256, 60000
    lens = [cached + new]
    cos, sin = tables(4, dh)
    c = make_cache(67, 1, dh, page, lens, DTYPES[dtype])
    table = c["table"][0]
    # scores: 8 q k = 20.3 ln 2 for the one key and 0 for the others, a little different for every token
    qkv = np.zeros((new, 3 * dh), np.float32)
    qkv[:, :dh] = (20.3 * np.log(2) / 8 * (1 + 0.03 * np.arange(new) / new))[:, None]
    slot = 7 if first else 31000
    pg, at = table[slot // page], slot % page
    k = np.zeros((len(table) * page, dh))
    v = np.ones((len(table) * page, dh)) * (1 + 0.25 * np.cos(np.arange(dh)))
    k[slot], v[slot] = 1.0, 0.0
    for name, x in (("k", k), ("v", v)):
        x = x.reshape(len(table), page, dh)
        if dtype == "i8":
            scale = np.maximum(np.abs(x).max(-1), 1e-30).astype(np.float32) / np.float32(127)
            c[name + "_scale"][table, 0] = scale
            c[name][table, 0, :, :dh] = np.clip(np.rint(x / scale[..., None]), -127, 127)
        else:
            c[name][table, 0, :, :dh] = x
    positions = np.zeros(new, np.int32)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, 1, None, new, lens, positions=positions)
    # (the oracle's own loop over the slots takes long at 80 tokens: its definition at once, tokens of one call being alike)
    kk, vv = (c[n][table, 0, :, :dh].astype(np.float64).reshape(-1, dh) for n in ("k", "v"))
    if dtype == "i8":
        kk, vv = kk * c["k_scale"][table, 0].astype(np.float64).reshape(-1, 1), vv * c["v_scale"][table, 0].astype(np.float64).reshape(-1, 1)
    want, reach = np.zeros((new, 1, dh)), np.zeros((new, 1))
    for i in range(new):
        n = cached + i + 1
        s = kk[:n] @ qkv[i, :dh].astype(np.float64) / 8
        p = np.exp(s - s.max())
        p /= p.sum()
        want[i, 0], reach[i, 0] = p @ vv[:n], (p @ np.abs(vv[:n])).max()
    # scores of 14 instead of 2: 22 bits of a product of the operands and fp32 sums, 2^-21 of it before the exponential
    check_each(got, want, (REL + 15 * 2.0 ** -21) * reach + 2.0 ** -37 * 1.25 * lens[0])


# ---------------------------------------------------------------- rows that are no numbers

@pytest.mark.parametrize("dh,hq,hkv,page", [(128, 4, 2, 32), (100, 2, 1, 16), (64, 2, 2, 64), (32, 4, 4, 16), (16, 1, 1, 16)])
def test_int8_rows_that_are_no_numbers(dh, hq, hkv, page):
    """A new row with an infinite or NaN component is stored as no number at all: codes of zero under a scale that is infinite or NaN.
    Every other row has the oracle's bits; tokens that see such a slot get no numbers either."""
    B, R = _mods()
    print("no numbers", dh, hq, hkv, page, flush=True)
    new, cached = 40, 10
    lens = [cached + new]
    cos, sin = tables(lens[0], dh)
    c = make_cache(69, hkv, dh, page, [cached], np.int8, table_pages=-(-lens[0] // page))
    qkv = synth.normal(69, dh, (new, (hq + 2 * hkv) * dh))
    rng = np.random.default_rng(dh)
    rows = qkv.reshape(new, hq + 2 * hkv, dh)
    bad = {}                                                      # (token, name, head) -> values planted
    for i, what in ((3, [np.nan]), (7, [np.inf]), (8, [-np.inf]), (15, [np.inf, np.nan]), (16, [np.nan, -np.inf, np.inf]), (38, [np.inf, np.inf])):
        for name, first in (("k", hq), ("v", hq + hkv)):
            h = int(rng.integers(hkv))
            rows[i, first + h, rng.permutation(dh)[:len(what)]] = what
            bad[i, name, h] = what
    want = {n: x.copy() for n, x in c.items()}
    with np.errstate(all="ignore"):
        K.append(want, qkv, hq, None, lens, None, cos, sin)
    g = OnGpu(B, R, c, dh, cos, sin)
    g.append(qkv, hq, None, new, lens)
    got = g.host()
    for (i, name, h), what in bad.items():
        slot = cached + i
        at = c["table"][0, slot // page], h, slot % page
        assert not got[name][at].any() and not np.isfinite(got[name + "_scale"][at]), (i, name, h, what)
        if name == "v":
            assert np.isnan(got["v_scale"][at]) == bool(np.isnan(what).any())
        for n in (name, name + "_scale"):
            got[n][at] = want[n][at] = 0
    for n in c:
        assert same_bits(got[n], want[n]), n
    out = g.attend(qkv, hq, None, new, lens).reshape(new, hq, dh)
    group = hq // hkv
    for i in range(new):
        for h in range(hq):
            sees = any(j <= i and x == h // group for j, _, x in bad)
            assert (np.isnan(out[i, h]).all() if sees else np.isfinite(out[i, h]).all()), (i, h)
