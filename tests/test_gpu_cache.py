"""GPU parity of the paged key/value cache: append, attention over it, selection, moving, and a run of all of them.

Bounds.  Append: the rotation's products and sums are rounded one by one on both sides, so rows are equal bit for bit.
Attention: the bound of the attention stage (a score is a sum of head_dim products carried with about 22 bits and summed in
fp32, a few 1e-7 sqrt(head_dim) before the exponential, hence a few 1e-6 on a probability and on the output, a convex
combination of value rows): 2e-6 of the largest |output| of a state for inputs of unit scale.  The cache's values are inputs here
(an fp16 or int8 row is what it stands for), so the bound does not depend on their type.  A weight is a sum of probabilities, each
with that relative error: 4e-6 of what was added, and one rounding of the running sum, 2^-24 of it, per addition (twice here).
An error of eps on every probability moves an output by at most eps sum_j p_j |v_j|, not by eps |output|: over thousands of
slots of either sign the output is small against the rows it is made of.  So the 2e-6 are of that sum (the oracle's `reach`).
Selection and moves are exact.

Slots and pages that no state owns, and what lies behind head_dim in a row, hold NaN wherever the type can.
"""
import numpy as np
import pytest

from oracle import bitrl_oracle as O
from oracle import cache_oracle as K
from paper_2604_24273_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

REL = 2e-6
DTYPES = {"f32": np.float32, "f16": np.float16, "i8": np.int8}


def _mods():
    from paper_2604_24273_amd import binding as B
    from paper_2604_24273_amd import runtime as R
    B.lib()
    return B, R


def tables(n, dh, theta=10000.0):
    inv = theta ** (-2.0 * np.arange(dh // 2) / dh)
    ang = np.arange(n)[:, None] * inv[None, :]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def make_cache(seed, hkv, dh, page, lens, dtype, spare=2, table_pages=None, scale=1.0):
    """A host cache whose slots below lens hold values, everything else NaN (or junk where the type has none)."""
    row = (dh + 15) // 16 * 16
    most = max(1, max(-(-n // page) for n in lens)) if table_pages is None else table_pages
    states = len(lens)
    pages = states * most + spare
    rng = np.random.default_rng(seed)
    c = {"table": rng.permutation(pages)[:states * most].astype(np.int32).reshape(states, most)}
    live = np.zeros((pages, page), dtype=bool)
    for b, n in enumerate(lens):
        for j in range(n):
            live[c["table"][b, j // page], j % page] = True
    for i, name in enumerate(("k", "v")):
        x = synth.normal(seed, 10 + i, (pages, hkv, page, row), scale)
        if dtype == np.int8:
            codes = np.clip(np.rint(x * (42 / scale)), -127, 127).astype(np.int8)
            codes.transpose(0, 2, 1, 3)[~live] = 99
            codes[..., dh:] = 77
            s = (0.8 + 0.4 * rng.random((pages, hkv, page))).astype(np.float32) * np.float32(scale / 42)
            s.transpose(0, 2, 1)[~live] = np.nan
            c[name], c[name + "_scale"] = codes, s
        else:
            x = x.astype(dtype)
            x.transpose(0, 2, 1, 3)[~live] = np.nan
            x[..., dh:] = np.nan
            c[name] = x
    return c


class OnGpu:
    def __init__(self, B, R, c, dh, cos, sin):
        self.B, self.R, self.dh = B, R, dh
        self.t = {n: R.dev(x) for n, x in c.items()}
        self.cos, self.sin = R.dev(cos), R.dev(sin)
        self.struct = B.make_kv_cache(self.t["k"], self.t["v"], self.t.get("k_scale"), self.t.get("v_scale"), self.t["table"], dh)

    def host(self):
        return {n: x.cpu().numpy() for n, x in self.t.items()}

    def ints(self, x):
        return None if x is None else self.R.dev(np.asarray(x, dtype=np.int32))

    def append(self, qkv, hq, cu, max_new, lens, positions=None):
        self.B.attention_cache_append(self.struct, self.R.dev(qkv), hq, qkv.shape[0], len(lens), self.ints(cu), max_new,
                                      self.ints(lens), self.ints(positions), self.cos, self.sin)

    def attend(self, qkv, hq, cu, max_new, lens, max_len=None, positions=None, tree=None, weights=None):
        T, hkv = qkv.shape[0], self.t["k"].shape[1]
        max_len = max(1, max(lens)) if max_len is None else max_len
        out = torch.full((T, hq * self.dh), float("nan"), device="cuda")
        need = self.B.brl_attention_cached_workspace_bytes(self.struct, hq, T, len(lens), max_new, max_len, weights is not None)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")          # NaN wherever it is read as a number
        tr = None if tree is None else self.R.dev(tree.view(np.int32))
        self.B.attention_cached_forward(self.struct, self.R.dev(qkv), hq, T, len(lens), self.ints(cu), max_new, self.ints(lens),
                                        max_len, self.ints(positions), self.cos, self.sin, tr, out, weights, ws)
        torch.cuda.synchronize()
        return out.cpu().numpy()


def same_bits(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and a.tobytes() == b.tobytes()


def check_rows(got, want, reach, cu, T, n_states, rel=REL):
    """Rows of every state within rel of the state's largest reach; rows of no state untouched."""
    worst = 0.0
    for b in range(n_states):
        r0, r1 = (b * T // n_states, (b + 1) * T // n_states) if cu is None else (cu[b], cu[b + 1])
        if r1 == r0:
            continue
        g, w = got[r0:r1].astype(np.float64), want[r0:r1]
        assert np.all(np.isfinite(g)), "state %d" % b
        worst = max(worst, np.abs(g - w).max() / max(reach[r0:r1].max(), 1e-30))
    print("   worst %.2e (bound %.1e)" % (worst, rel), flush=True)
    assert worst <= rel
    if cu is not None:
        assert np.all(np.isnan(got[cu[-1]:]))


def ancestors(rng, new, words):
    """A random tree: token i hangs on an earlier token or on the prefix."""
    m = np.zeros((new, words), dtype=np.uint32)
    for i in range(new):
        p = int(rng.integers(-1, i))
        if p >= 0:
            m[i] = m[p]
        m[i, i // 32] |= np.uint32(1 << (i % 32))
    return m


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", [
    (128, 20, 5, 32, [200], [1]),
    (128, 8, 2, 16, [0, 15, 16, 17, 40], [1, 3, 0, 40, 7]),
    (100, 4, 4, 64, [63, 0, 5], [2, 64, 130]),
    (100, 2, 1, 16, [14, 3], [20, 1]),
    (64, 4, 2, 128, [5, 127], [9, 2]),
    (32, 8, 8, 256, [0, 300], [33, 1]),
    (16, 8, 1, 16, [9, 0, 31, 2], [1, 1, 2, 100]),
])
def test_append_writes_the_oracles_bits_and_nothing_else(dh, hq, hkv, page, cached, new, dtype):
    B, R = _mods()
    print("append", dh, hq, hkv, page, cached, new, dtype, flush=True)
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + 2                                                   # two rows of no state
    qkv = synth.normal(3, dh + page, (T, (hq + 2 * hkv) * dh))
    qkv[0, hq * dh:(hq + hkv) * dh] = 0                                     # a row of zeros
    cos, sin = tables(700, dh)
    c = make_cache(4, hkv, dh, page, cached, DTYPES[dtype], table_pages=max(-(-n // page) for n in lens) + 1)
    rng = np.random.default_rng(5)
    for positions in (None, rng.integers(-3, 720, T)):                    # positions past the table count as its ends
        g = OnGpu(B, R, c, dh, cos, sin)
        g.append(qkv, hq, cu, max(new), lens, positions)
        want = {n: x.copy() for n, x in c.items()}
        K.append(want, qkv, hq, cu, lens, positions, cos, sin)
        got = g.host()
        for n in c:
            assert same_bits(got[n], want[n]), n


def test_append_uniform_batches_and_tokens_without_a_slot():
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 64, 16
    cos, sin = tables(100, dh)
    c = make_cache(6, hkv, dh, page, [0, 0, 0], np.float32, table_pages=2)
    qkv = synth.normal(6, 1, (15, (hq + 2 * hkv) * dh))
    for lens in ([5, 20, 32], [3, -7, 4000], [0, 5, 2]):     # fewer slots than tokens; negative; past the table
        g = OnGpu(B, R, c, dh, cos, sin)
        g.append(qkv, hq, None, 5, lens)
        want = {n: x.copy() for n, x in c.items()}
        K.append(want, qkv, hq, None, [min(max(n, 0), 32) for n in lens], None, cos, sin)
        got = g.host()
        for n in c:
            assert same_bits(got[n], want[n]), (n, lens)


# ---------------------------------------------------------------- attention

ATTEND = [
    # (head_dim, heads, kv heads, page, cached, new)
    (128, 20, 5, 32, [300], [1]),
    (128, 20, 5, 64, [0], [1]),                                   # its own key only
    (128, 8, 2, 16, [31, 32, 33, 0, 500], [1, 1, 1, 1, 1]),
    (128, 4, 1, 128, [5000], [1]),                                # split along the keys
    (128, 16, 1, 32, [700, 64], [2, 1]),                          # 16 heads to a group
    (128, 4, 4, 64, [100, 7], [40, 33]),
    (128, 8, 2, 32, [0, 0, 0], [130, 1, 64]),                     # prompts
    (100, 4, 4, 64, [130, 0, 63], [3, 70, 1]),
    (100, 2, 1, 16, [47], [5]),
    (64, 4, 2, 256, [300, 1], [9, 20]),
    (64, 12, 4, 32, [40, 0, 90, 12], [0, 8, 17, 0]),              # states without new tokens; groups of three
    (32, 8, 8, 64, [100, 31], [33, 2]),
    (16, 8, 1, 16, [100, 0, 17, 64], [1, 16, 5, 40]),
    # blocks of all states shared evenly among workgroups, states cut anywhere
    (64, 4, 2, 32, [1500, 3, 0, 2000, 700, 31], [1, 1, 0, 2, 1, 1]),
    (128, 5, 1, 64, [2500, 0, 1100], [3, 6, 1]),                  # two row tiles
    # many rows and long keys: the keys split among workgroups
    (128, 8, 2, 64, [700], [12]),
    (100, 3, 3, 32, [900, 40, 0], [70, 2, 0]),
    (32, 4, 2, 16, [1300], [50]),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", ATTEND)
def test_attention_over_the_cache_against_the_oracle(dh, hq, hkv, page, cached, new, mask, dtype):
    B, R = _mods()
    print("attend", dh, hq, hkv, page, cached, new, mask, dtype, flush=True)
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + 1
    rng = np.random.default_rng(dh + sum(cached))
    qkv = synth.normal(7, dh + T, (T, (hq + 2 * hkv) * dh))
    cos, sin = tables(max(lens) + 40, dh, 500000.0 if dh == 128 else 10000.0)
    c = make_cache(8, hkv, dh, page, lens, DTYPES[dtype])
    positions = rng.integers(0, max(lens) + 40, T)
    words = -(-max(new) // 32)
    tree = None if mask == "causal" else np.concatenate([ancestors(rng, n, words) for n in new] + [np.zeros((1, words), np.uint32)])
    g = OnGpu(B, R, c, dh, cos, sin)
    hkv_w = torch.rand(len(lens), hkv, max(lens) + 3, device="cuda")
    before = hkv_w.cpu().numpy().copy()
    got = g.attend(qkv, hq, cu, max(new), lens, positions=positions, tree=tree, weights=hkv_w)
    want, added, reach = K.attend(c, qkv, hq, cu, lens, positions, cos, sin, tree)
    check_rows(got, want, reach, cu, T, len(lens))
    w = hkv_w.cpu().numpy()
    longest = added.shape[2]
    err = np.abs(w[:, :, :longest].astype(np.float64) - before[:, :, :longest] - added)
    assert np.all(err <= 4e-6 * added + 2.0 ** -23 * w[:, :, :longest])
    assert same_bits(w[:, :, longest:], before[:, :, longest:])
    # without weights, and with room to spare in the bounds: the same within the bound
    again = g.attend(qkv, hq, cu, T, lens, max_len=c["table"].shape[1] * page, positions=positions, tree=tree)
    check_rows(again, want, reach, cu, T, len(lens))
    for n, x in g.host().items():
        assert same_bits(x, c[n]), n


@pytest.mark.parametrize("states", [63, 64, 65, 130, 300])
def test_many_states_of_very_different_length(states):
    """The shared list of blocks over more states than a wavefront has lanes: most hold little or nothing, a few a great deal."""
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 32, 16
    rng = np.random.default_rng(states)
    lens = [int(x) for x in rng.integers(0, 60, states)]
    for b, n in ((0, 1200), (states - 1, 1700), (states // 2, 1057)):
        lens[b] = n
    new = [int(x) for x in rng.integers(0, 3, states)]
    new[0] = new[-1] = 1
    lens = [max(a, n) if a % 7 else a for a, n in zip(lens, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + 1
    cos, sin = tables(1800, dh)
    c = make_cache(23, hkv, dh, page, lens, np.float16)
    qkv = synth.normal(23, states, (T, (hq + 2 * hkv) * dh))
    w = torch.zeros(states, hkv, 1700, device="cuda")
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, 2, lens, weights=w)
    want, added, reach = K.attend(c, qkv, hq, cu, lens, None, cos, sin)
    check_rows(got, want, reach, cu, T, states)
    assert np.all(np.abs(w.cpu().numpy() - added) <= 4e-6 * added)


def test_rows_that_see_nothing_are_zeros():
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 128, 32
    cos, sin = tables(100, dh)
    lens = [5, 45, 0, 3, -4]
    new = [5, 40, 2, 6, 2]                  # nothing cached; some cached; no slot at all; more tokens than slots; lens below zero
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1])
    c = make_cache(9, hkv, dh, page, [max(n, 0) for n in lens], np.float32)
    qkv = synth.normal(9, 1, (T, (hq + 2 * hkv) * dh))
    tree = np.zeros((T, 2), np.uint32)
    tree[2, 0] = 1 << 1
    tree[cu[3]:cu[4], 0] = 0b111111          # tokens without a slot are not there to be seen
    clamped = [max(n, 0) for n in lens]
    c["table"] = np.concatenate([c["table"], np.zeros((5, 128), np.int32)], axis=1)
    for t in (tree, None):
        want, added, reach = K.attend(c, qkv, hq, cu, clamped, None, cos, sin, t)
        empty = np.all(want == 0, axis=1)
        for bound in (64, 4000):                             # short and long bounds on the slots take different forms
            w = torch.zeros(5, hkv, bound, device="cuda")
            got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, max_len=bound, tree=t, weights=w)
            check_rows(got, want, reach, cu, T, 5)
            assert empty.any() and np.all(got[empty] == 0)
            assert np.abs(w.cpu().numpy()[:, :, :added.shape[2]] - added).max() <= 4e-6 * max(1.0, added.max())
    # the same for few rows
    few = [1, 1, 2, 2, 1]
    cu = np.concatenate([[0], np.cumsum(few)]).astype(np.int32)
    T = int(cu[-1])
    for t in (np.zeros((T, 1), np.uint32), None):
        want, added, reach = K.attend(c, qkv[:T], hq, cu, clamped, None, cos, sin, t)
        for bound in (64, 4000):
            w = torch.zeros(5, hkv, bound, device="cuda")
            got = OnGpu(B, R, c, dh, cos, sin).attend(qkv[:T], hq, cu, 2, lens, max_len=bound, tree=t, weights=w)
            check_rows(got, want, reach, cu, T, 5)
            empty = np.all(want == 0, axis=1)
            assert empty.any() and np.all(got[empty] == 0)
            assert np.abs(w.cpu().numpy()[:, :, :added.shape[2]] - added).max() <= 4e-6 * max(1.0, added.max())


def test_mask_words_short_of_the_new_tokens():
    """Tokens past the last word of the mask are seen by nobody, not even by themselves."""
    B, R = _mods()
    hq, hkv, dh = 2, 2, 32
    cos, sin = tables(100, dh)
    c = make_cache(10, hkv, dh, 16, [60], np.float16)
    qkv = synth.normal(10, 1, (40, 6 * dh))
    tree = np.full((40, 1), 0xffffffff, np.uint32)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, None, 40, [60], tree=tree)
    want, _, reach = K.attend(c, qkv, hq, None, [60], None, cos, sin, tree)
    check_rows(got, want, reach, None, 40, 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("new", [1, 70])
def test_pages_outside_the_pool_disappear(dtype, new):
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 64, 16
    cos, sin = tables(300, dh)
    lens = [200, 100]
    c = make_cache(11, hkv, dh, page, lens, DTYPES[dtype])
    c["table"][0, 2], c["table"][0, 7], c["table"][1, 0] = -1, c["k"].shape[0], 2 ** 31 - 1
    c["table"][0, 12] = -2 ** 31
    qkv = synth.normal(11, 1, (2 * new, (hq + 2 * hkv) * dh))
    g = OnGpu(B, R, c, dh, cos, sin)
    w = torch.zeros(2, hkv, 200, device="cuda")
    got = g.attend(qkv, hq, None, new, lens, weights=w)
    want, added, reach = K.attend(c, qkv, hq, None, lens, None, cos, sin)
    check_rows(got, want, reach, None, 2 * new, 2)
    assert np.abs(w.cpu().numpy() - added).max() <= 4e-6 * added.max()
    g.append(qkv, hq, None, new, lens)
    ref = {n: x.copy() for n, x in c.items()}
    K.append(ref, qkv, hq, None, lens, None, cos, sin)
    for n, x in g.host().items():
        assert same_bits(x, ref[n]), n


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_large_and_small_values(dtype):
    """Scores that span hundreds of units; value rows of very different size; keys near the largest fp16."""
    B, R = _mods()
    hq, hkv, dh, page = 4, 1, 128, 32
    cos, sin = tables(300, dh)
    lens = [290, 40]
    c = make_cache(12, hkv, dh, page, lens, DTYPES[dtype], scale=3.0)
    qkv = synth.normal(12, 1, (6, (hq + 2 * hkv) * dh), 3.0)
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, None, 3, lens)
    want, _, reach = K.attend(c, qkv, hq, None, lens, None, cos, sin)
    check_rows(got, want, reach, None, 6, 2, rel=9 * REL)                # three times the inputs: nine times the range of scores
    for b in range(2):
        c["k"][c["table"][b, 0], :, 3, :dh] = 60000.0               # a key that dwarfs all others, for one sign of the query's sum
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, None, 3, lens)
    want, _, reach = K.attend(c, qkv, hq, None, lens, None, cos, sin)
    assert np.all(np.isfinite(got)) and np.abs(got - want).max() <= 9 * REL * reach.max()


@pytest.mark.parametrize("scale", [1e-6, 1.0, 3e4])
def test_int8_scales_of_any_size(scale):
    """The rows' scales far from one and, within a state, six orders apart: the output follows the largest of them."""
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 128, 16
    cos, sin = tables(300, dh)
    lens = [200, 33]
    c = make_cache(13, hkv, dh, page, lens, np.int8)
    c["v_scale"] *= np.float32(scale / 100)
    for new in (1, 33):
        qkv = synth.normal(13, new, (2 * new, (hq + 2 * hkv) * dh))
        for spread in (False, True):
            d = {n: x.copy() for n, x in c.items()}
            if spread:
                d["v_scale"][::2] *= np.float32(1e-6)
            got = OnGpu(B, R, d, dh, cos, sin).attend(qkv, hq, None, new, lens)
            want, _, reach = K.attend(d, qkv, hq, None, lens, None, cos, sin)
            check_rows(got, want, reach, None, 2 * new, 2)


def test_rows_behind_four_gigabytes():
    """Offsets past 32 bits: bytes, elements and rows of the last pages of a large pool."""
    B, R = _mods()
    hq, hkv, dh, page = 4, 2, 128, 256
    pages = 40000                                      # 40000 * 2 * 256 * 128 * 2 bytes = 5.2 GB each
    cos, sin = tables(600, dh)
    small = make_cache(14, hkv, dh, page, [500], np.float16)
    ids = np.array([[pages - 1, pages - 3]], np.int32)
    k = torch.empty(pages, hkv, page, dh, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    for j in range(2):
        k[ids[0, j]] = torch.from_numpy(small["k"][small["table"][0, j]]).cuda()
        v[ids[0, j]] = torch.from_numpy(small["v"][small["table"][0, j]]).cuda()
    table = R.dev(ids)
    struct = B.make_kv_cache(k, v, None, None, table, dh)
    tcos, tsin = R.dev(cos), R.dev(sin)
    for new in (1, 80):
        lens = R.dev(np.array([500], np.int32))
        qkv = synth.normal(14, new, (new, (hq + 2 * hkv) * dh))
        x, out = R.dev(qkv), torch.empty(new, hq * dh, device="cuda")
        ref = {n: a.copy() for n, a in small.items()}
        K.append(ref, qkv, hq, None, [500], None, cos, sin)
        B.attention_cache_append(struct, x, hq, new, 1, None, new, lens, None, tcos, tsin)
        w = torch.rand(1, hkv, 512, device="cuda")
        ws = R.device_bytes(B.brl_attention_cached_workspace_bytes(struct, hq, new, 1, new, 512, True))
        B.attention_cached_forward(struct, x, hq, new, 1, None, new, lens, 512, None, tcos, tsin, None, out, w, ws)
        want, _, reach = K.attend(ref, qkv, hq, None, [500], None, cos, sin)
        check_rows(out.cpu().numpy(), want, reach, None, new, 1)
        small = ref
    kept = np.sort(np.random.default_rng(1).permutation(500)[:100]).astype(np.int32).reshape(1, 1, 100)
    B.attention_cache_compact(struct, 1, lens, 512, R.dev(kept), 1, None, R.dev(np.array([100], np.int32)), None)
    K.compact(small, [500], kept, None, [100])
    for j in range(2):
        for name, t in (("k", k), ("v", v)):
            got, ref = t[ids[0, j]].cpu().numpy(), small[name][small["table"][0, j]]
            assert same_bits(got[:, :244, :dh], ref[:, :244, :dh]), name


def test_another_stream_and_graphs_that_share_a_workspace():
    """Work on a side stream; two captured steps with one workspace, replayed between eager calls."""
    B, R = _mods()
    hq, hkv, dh, page = 8, 2, 128, 64
    cos, sin = tables(3000, dh)
    lens = [2500, 900]
    c = make_cache(15, hkv, dh, page, lens, np.float16)
    g = OnGpu(B, R, c, dh, cos, sin)
    plans = []
    for new in (1, 40):
        qkv = synth.normal(15, new, (2 * new, (hq + 2 * hkv) * dh))
        plans.append({"new": new, "x": R.dev(qkv), "out": torch.zeros(2 * new, hq * dh, device="cuda"),
                      "w": torch.zeros(2, hkv, 2500, device="cuda"), "want": g.attend(qkv, hq, None, new, lens)})
    need = max(B.brl_attention_cached_workspace_bytes(g.struct, hq, 2 * p["new"], 2, p["new"], 2500, True) for p in plans)
    ws, dl = R.device_bytes(need), g.ints(lens)

    def step(p):
        B.attention_cached_forward(g.struct, p["x"], hq, 2 * p["new"], 2, None, p["new"], dl, 2500, None, g.cos, g.sin, None, p["out"],
                                   p["w"], ws)

    side = torch.cuda.Stream()
    for p in plans:
        with torch.cuda.stream(side):
            p["out"].zero_()
            step(p)
        side.synchronize()
        p["eager"], p["added"] = p["out"].clone(), p["w"].clone()
        assert np.abs(p["eager"].cpu().numpy() - p["want"]).max() <= 2 * REL      # (reach: about the mean |v|, under one)
        p["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(p["graph"]):
            step(p)
    for rep in range(3):
        for p in plans:
            p["out"].fill_(float("nan"))
            p["w"].zero_()
            ws.fill_(255)
            p["graph"].replay()
            torch.cuda.synchronize()
            assert torch.equal(p["out"], p["eager"]) and torch.equal(p["w"], p["added"]), rep
            step(plans[0])
            torch.cuda.synchronize()


def test_a_captured_step_follows_the_lengths_on_the_device():
    """One captured decode step serves a growing state: lens, positions and tokens are read on the device."""
    B, R = _mods()
    hq, hkv, dh, page = 4, 1, 64, 16
    cos, sin = tables(200, dh)
    c = make_cache(16, hkv, dh, page, [30], np.float32, table_pages=8)
    g = OnGpu(B, R, c, dh, cos, sin)
    x, out = torch.zeros(1, (hq + 2 * hkv) * dh, device="cuda"), torch.zeros(1, hq * dh, device="cuda")
    dl = g.ints([30])
    ws = R.device_bytes(B.brl_attention_cached_workspace_bytes(g.struct, hq, 1, 1, 1, 128, False))

    def step():
        dl.add_(1)
        B.attention_cache_append(g.struct, x, hq, 1, 1, None, 1, dl, None, g.cos, g.sin)
        B.attention_cached_forward(g.struct, x, hq, 1, 1, None, 1, dl, 128, None, g.cos, g.sin, None, out, None, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    dl.copy_(g.ints([30]))
    for i in range(40):
        row = synth.normal(16, 50 + i, (1, (hq + 2 * hkv) * dh))
        x.copy_(R.dev(row))
        graph.replay()
        torch.cuda.synchronize()
        K.append(c, row, hq, None, [31 + i], None, cos, sin)
        want, _, reach = K.attend(c, row, hq, None, [31 + i], None, cos, sin)
        check_rows(out.cpu().numpy(), want, reach, None, 1, 1)


@pytest.mark.parametrize("dh,hq,hkv,theta", [(128, 20, 5, 500000.0), (100, 4, 4, 10000.0), (16, 8, 1, 10000.0)])
def test_an_fp32_cache_gives_what_whole_states_give(dh, hq, hkv, theta):
    """attention_forward on whole states against append and attention in pieces, rotary table from the library."""
    B, R = _mods()
    lens = [150, 37, 64]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    qkv = synth.normal(17, dh, (int(cu[-1]), (hq + 2 * hkv) * dh))
    cos, sin = torch.zeros(200, dh // 2, device="cuda"), torch.zeros(200, dh // 2, device="cuda")
    B.attention_rope_table(cos, sin, dh, theta)
    hc, hs = tables(200, dh, theta)
    assert np.abs(cos.cpu().numpy() - hc).max() <= 2.0 ** -23 and np.abs(sin.cpu().numpy() - hs).max() <= 2.0 ** -23
    whole = torch.zeros(int(cu[-1]), hq * dh, device="cuda")
    ws = R.device_bytes(B.brl_attention_workspace_bytes(3, 150, hq, hkv, dh))
    B.attention_forward(R.dev(qkv), 3, 150, R.dev(cu), cu, hq, hkv, dh, theta, B.BRL_ATTN_MFMA, whole, ws)
    whole = whole.cpu().numpy()
    c = make_cache(17, hkv, dh, 32, [0, 0, 0], np.float32, table_pages=5)
    g = OnGpu(B, R, c, dh, cos.cpu().numpy(), sin.cpu().numpy())
    done = [0, 0, 0]
    for step in ([100, 30, 1], [1, 0, 62], [49, 7, 1]):
        rows = np.concatenate([qkv[cu[b] + done[b]:cu[b] + done[b] + n] for b, n in enumerate(step)])
        part = np.concatenate([whole[cu[b] + done[b]:cu[b] + done[b] + n] for b, n in enumerate(step)])
        done = [d + n for d, n in zip(done, step)]
        scu = np.concatenate([[0], np.cumsum(step)]).astype(np.int32)
        g.append(rows, hq, scu, max(step), done)
        got = g.attend(rows, hq, scu, max(step), done)
        assert np.abs(got - part).max() <= 2 * REL * np.abs(part).max()


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", [
    (128, 4, 4, 16, [40, 0, 3], [9, 5, 16]),
    (128, 20, 5, 32, [1700, 31], [3, 2]),                         # the shared list
    (100, 2, 1, 64, [700, 90, 0], [7, 8, 1]),
    (16, 8, 2, 16, [20], [4]),
    (64, 4, 2, 32, [100, 0], [40, 20]),                           # keys shared by many rows
    (100, 3, 3, 32, [900], [70]),                                 # and split
    (128, 8, 2, 64, [10, 0], [130, 33]),                          # two row tiles per wavefront
    (32, 12, 4, 128, [0], [200]),
])
def test_infinities_and_nan_stay_with_the_tokens_that_see_them(dh, hq, hkv, page, cached, new, mask, dtype):
    """New tokens whose values (int8: the scale of a value row) or keys are infinite or NaN: a token that does not see their slots
    gets what it gets without them; one that does has the components not finite that the sum says.  (What a token gets that sees an
    infinite key is open: an operand's two halves times infinity can be infinities of either sign.  Keys: the tokens that see none.)"""
    B, R = _mods()
    print("strange", dh, hq, hkv, page, cached, new, mask, dtype, flush=True)
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1])
    rng = np.random.default_rng(dh + T)
    qkv = synth.normal(31, dh + T, (T, (hq + 2 * hkv) * dh))
    cos, sin = tables(max(lens), dh)
    words = -(-max(new) // 32)
    tree = None if mask == "causal" else np.concatenate([ancestors(rng, n, words) for n in new])
    for name in ("v", "k"):
        c = make_cache(32, hkv, dh, page, lens, DTYPES[dtype])
        for b, n in enumerate(new):
            for i, bad in ((n // 2, np.inf), (n - 1, np.nan), (2 * n // 3, -np.inf)):
                slot = cached[b] + i
                pg, at, h = c["table"][b, slot // page], slot % page, i % hkv
                if dtype == "i8":
                    c[name + "_scale"][pg, h, at] = bad
                else:
                    c[name][pg, h, at, rng.integers(0, dh, 3)] = bad
        ref = dict(c)
        if name == "k":                                                   # NaN, which every token that sees it has in all components
            n = "k_scale" if dtype == "i8" else "k"
            ref[n] = np.where(np.isinf(c[n]), c[n].dtype.type(np.nan), c[n])
        with np.errstate(all="ignore"):
            want, added, reach = K.attend(ref, qkv, hq, cu, lens, None, cos, sin, tree)
        w = torch.zeros(len(lens), hkv, max(lens), device="cuda")
        got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, tree=tree, weights=w)
        plain = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, tree=tree)
        finite = np.isfinite(want)
        assert finite.any() and not finite.all()
        # reach of rows with something infinite is no bound for their finite components: the largest value there is
        most = 127 * 1.2 / 42 if dtype == "i8" else max(np.abs(c["v"][np.isfinite(c["v"])].astype(np.float64)).max(), 1.0)
        bound = REL * np.where(np.isfinite(reach), reach, most)[:, None]
        for y in (got, plain):
            assert np.all(np.isfinite(y)[finite]) and (name == "k" or np.array_equal(np.isfinite(y), finite)), name
            diff = np.abs(y[finite].astype(np.float64) - want[finite])
            assert np.all(diff <= np.broadcast_to(np.maximum(bound, REL * most), want.shape)[finite]), name
        if name == "v":
            g = w.cpu().numpy()[:, :, :added.shape[2]]
            assert np.all(np.abs(g - added) <= 4e-6 * added + 2.0 ** -23 * g)


# ---------------------------------------------------------------- selection and moving

@pytest.mark.parametrize("lens,keep,first,recent", [
    ([0, 1, 5, 6, 7, 100], 6, 1, 2),
    ([100, 99], 6, 6, 0), ([100, 8], 6, 0, 6), ([50], 6, 2, 4),         # nothing chosen by weight
    ([5000, 1024, 1025, 3], 1000, 4, 100),
    ([4097, 2048], 1, 0, 0),
    ([2000], 1999, 0, 0),
    ([70001, 65536, 65537], 20000, 4, 5000),
    ([140000], 139000, 7, 11),
])
def test_select_against_the_oracle(lens, keep, first, recent):
    B, R = _mods()
    print("select", lens, keep, first, recent, flush=True)
    hkv, most = 3, max(lens)
    w = np.exp(1.5 * synth.normal(18, keep, (len(lens), hkv, most + 5))).astype(np.float32)
    w[:, 0] = np.round(w[:, 0], 1)                                        # many ties
    w[:, 1, ::3] = 0
    w[:, 2] -= 1
    special = np.array([np.nan, np.inf, -np.inf, -0.0, 0.0, 1e-45, -1e-45, 3e38], np.float32)
    w[:, 2, :most // 2 * 2:max(1, most // 40)] = np.resize(special, w[:, 2, :most // 2 * 2:max(1, most // 40)].shape)
    kept = torch.full((len(lens), hkv, keep), 7, dtype=torch.int32, device="cuda")
    counts = torch.full((len(lens),), 7, dtype=torch.int32, device="cuda")
    B.attention_cache_select(R.dev(w), len(lens), hkv, R.dev(np.array(lens, np.int32)), most, keep, first, recent, kept, counts)
    want, n = K.select(w, lens, keep, first, recent)
    assert np.array_equal(counts.cpu().numpy(), n)
    assert np.array_equal(kept.cpu().numpy(), want)


def test_select_when_all_weights_are_alike():
    B, R = _mods()
    for value in (0.0, np.nan, 1.0, np.inf):
        w = np.full((2, 2, 3000), value, np.float32)
        kept = torch.zeros(2, 2, 700, dtype=torch.int32, device="cuda")
        counts = torch.zeros(2, dtype=torch.int32, device="cuda")
        lens = [2999, 5000]                                               # the second counts as max_len
        B.attention_cache_select(R.dev(w), 2, 2, R.dev(np.array(lens, np.int32)), 3000, 700, 3, 50, kept, counts)
        want, n = K.select(w, [2999, 3000], 700, 3, 50)
        assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("dh,hkv,page,lens,counts,start,shared", [
    (128, 5, 32, [500, 64, 33], [200, 64, 1], None, False),
    (128, 2, 16, [1000], [999], None, False),                             # everything moves by at most one
    (100, 4, 64, [300, 17, 0], [100, 0, 0], None, False),
    (64, 2, 256, [700, 900], [50, 300], [600, 100], True),                # an accepted branch at the tail
    (32, 8, 64, [2000, 5], [900, 5], None, True),
    (16, 1, 16, [4000, 100], [1500, 99], [10, 0], False),
    (16, 3, 128, [12000], [9000], None, False),
])
def test_compact_against_the_oracle(dh, hkv, page, lens, counts, start, shared, dtype):
    B, R = _mods()
    print("compact", dh, hkv, page, lens, counts, start, shared, dtype, flush=True)
    c = make_cache(19, hkv, dh, page, lens, DTYPES[dtype])
    rng = np.random.default_rng(dh + page)
    heads = 1 if shared else hkv
    ld = max(counts) + 3
    kept = np.full((len(lens), heads, ld), -1, np.int32)
    for b, n in enumerate(lens):
        s0 = 0 if start is None else start[b]
        for h in range(heads):
            kept[b, h, :counts[b]] = s0 + np.sort(rng.permutation(n - s0)[:counts[b]])
    w = rng.random((len(lens), hkv, max(lens) + 2)).astype(np.float32)
    cos, sin = tables(4, dh)
    for weights in (False, True):
        g = OnGpu(B, R, c, dh, cos, sin)
        tw = R.dev(w) if weights else None
        B.attention_cache_compact(g.struct, len(lens), g.ints(lens), max(lens), R.dev(kept), heads, g.ints(start), g.ints(counts), tw)
        want, ww = {n: x.copy() for n, x in c.items()}, w.copy()
        K.compact(want, lens, kept, start, counts, ww if weights else None)
        for n, x in g.host().items():
            assert same_bits(x, want[n]), n
        if weights:
            assert same_bits(tw.cpu().numpy(), ww)


def test_compact_ignores_what_is_not_there():
    """Entries below their target, repeated, past the state, of pages outside the pool; counts and starts out of range."""
    B, R = _mods()
    hkv, dh, page = 2, 32, 16
    lens = [100, 100, 40]
    c = make_cache(20, hkv, dh, page, lens, np.float16)
    c["table"][1, 3], c["table"][1, 0] = -5, 10 ** 6
    kept = np.zeros((3, hkv, 50), np.int32)
    kept[0, :] = np.sort(np.resize([3, 3, 3, 50, 99, 100, 10 ** 9], 50))
    kept[0, 1] = np.resize([-1, -10 ** 9, 0, 0, 20], 50)
    kept[1, :] = np.arange(50) + 40
    kept[2, :] = np.arange(50)
    counts, start = [1000, 50, -3], [0, 7, 10 ** 9]
    cos, sin = tables(4, dh)
    g = OnGpu(B, R, c, dh, cos, sin)
    before = g.host()
    B.attention_cache_compact(g.struct, 3, g.ints(lens), 100, R.dev(kept), hkv, g.ints(start), g.ints(counts), None)
    want = {n: x.copy() for n, x in c.items()}
    only = kept.copy()
    K.compact(want, lens, only, start, counts)
    got = g.host()
    assert same_bits(got["k"], want["k"]) and same_bits(got["v"], want["v"])
    assert same_bits(before["table"], got["table"])


# ---------------------------------------------------------------- all of them, as they are used

@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
def test_an_episode_prompt_steps_branches_eviction(dtype):
    """Prompts, steps with weights, eviction, a tree of candidates, its accepted branch, further steps: every output against
    the oracle run on the same calls."""
    B, R = _mods()
    hq, hkv, dh, page, keep = 8, 2, 64, 16, 60
    theta = 10000.0
    cos, sin = tables(400, dh, theta)
    c = make_cache(21, hkv, dh, page, [0, 0], DTYPES[dtype], table_pages=10)
    g = OnGpu(B, R, c, dh, cos, sin)
    ref = {n: x.copy() for n, x in c.items()}
    rng = np.random.default_rng(21)
    lens, seen = [0, 0], [0, 0]
    gw, rw = torch.zeros(2, hkv, 160, device="cuda"), np.zeros((2, hkv, 160))
    turn = [0]

    def attend(new, depths=None, tree=None, grow=True):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1])
        turn[0] += 1
        qkv = synth.normal(22, turn[0], (T, (hq + 2 * hkv) * dh))
        total = [a + n for a, n in zip(lens, new)]
        pos = np.concatenate([seen[b] + (np.arange(n) if depths is None else depths[b]) for b, n in enumerate(new)])
        g.append(qkv, hq, cu, max(new), total, pos)
        K.append(ref, qkv, hq, cu, total, pos, cos, sin)
        got = g.attend(qkv, hq, cu, max(new), total, max_len=160, positions=pos, tree=tree, weights=gw)
        want, added, reach = K.attend(ref, qkv, hq, cu, total, pos, cos, sin, tree)
        rw[:, :, :added.shape[2]] += added
        check_rows(got, want, reach, cu, T, 2)
        for n, x in g.host().items():
            assert same_bits(x, ref[n]), n
        lens[:] = total
        if grow:
            seen[:] = [s + n for s, n in zip(seen, new)]

    attend([70, 40])
    for _ in range(3):
        attend([1, 1])
    attend([10, 20])
    # eviction: by the GPU's own sums (the oracle's differ in the last bits), so both sides move the same rows
    kept = torch.zeros(2, hkv, keep, dtype=torch.int32, device="cuda")
    counts = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert np.abs(gw.cpu().numpy() - rw).max() <= 1e-5 * rw.max()
    host_w = gw.cpu().numpy().copy()
    B.attention_cache_select(gw, 2, hkv, g.ints(lens), 160, keep, 4, 16, kept, counts)
    want_kept, want_counts = K.select(host_w, lens, keep, 4, 16)
    assert np.array_equal(kept.cpu().numpy(), want_kept) and np.array_equal(counts.cpu().numpy(), want_counts)
    B.attention_cache_compact(g.struct, 2, g.ints(lens), 160, kept, hkv, None, counts, gw)
    K.compact(ref, lens, want_kept, None, want_counts, host_w)
    assert same_bits(gw.cpu().numpy(), host_w)
    for n, x in g.host().items():
        assert same_bits(x, ref[n]), n
    lens[:] = [int(x) for x in want_counts]
    for b in range(2):
        gw[b, :, lens[b]:] = 0
    rw[:] = gw.cpu().numpy()
    attend([1, 2])
    # three candidates of three tokens each behind one state, two of two behind the other
    parents = [[-1, 0, 1, -1, 3, 4, -1, 6, 7], [-1, 0, -1, 2]]
    masks, depths = [], []
    for ps in parents:
        m, d = np.zeros((len(ps), 1), np.uint32), np.zeros(len(ps), np.int64)
        for i, p in enumerate(ps):
            if p >= 0:
                m[i], d[i] = m[p], d[p] + 1
            m[i, 0] |= np.uint32(1 << i)
        masks.append(m)
        depths.append(d)
    base = list(lens)
    attend([9, 4], depths=depths, tree=np.concatenate(masks), grow=False)
    # the second candidate of each is taken: its tokens move behind the prefix
    branch = np.array([[[base[0] + 3, base[0] + 4, base[0] + 5]], [[base[1] + 2, base[1] + 3, -1]]], np.int32)
    B.attention_cache_compact(g.struct, 2, g.ints(lens), 160, R.dev(branch), 1, g.ints(base), g.ints([3, 2]), gw)
    host_w = rw.copy()
    K.compact(ref, lens, branch, base, [3, 2], host_w)
    rw[:] = host_w
    for n, x in g.host().items():
        assert same_bits(x, ref[n]), n
    lens[:] = [base[0] + 3, base[1] + 2]
    seen[:] = [seen[0] + 3, seen[1] + 2]
    for b in range(2):
        gw[b, :, lens[b]:] = 0
        rw[b, :, lens[b]:] = 0
    attend([1, 30])
    attend([1, 1])
    assert np.abs(gw.cpu().numpy() - rw).max() <= 1e-5 * rw.max()


# ---------------------------------------------------------------- the holder

@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
def test_the_holder_through_an_episode(dtype):
    """runtime.KVCache with fewer pages than its states could fill: pages freed by one state are given to another; every output against
    the oracle on the cache's own arrays, every stored row against the oracle's."""
    B, R = _mods()
    hq, hkv, dh, page, theta = 6, 2, 64, 16, 10000.0
    kv = R.KVCache(3, hq, hkv, dh, 150, theta, dtype={"f32": torch.float32, "f16": torch.float16, "i8": torch.int8}[dtype], page_tokens=page,
                   n_pages=17, max_position=300, track_weights=True)
    for x in (kv.k, kv.v, kv.k_scale, kv.v_scale):
        if x is not None:
            x.fill_(7 if x.dtype == torch.int8 else float("nan"))
    cos, sin = kv.rope_cos.cpu().numpy(), kv.rope_sin.cpu().numpy()
    c64, s64 = tables(300, dh, theta)
    assert np.abs(cos - c64).max() < 1e-6 and np.abs(sin - s64).max() < 1e-6
    rw, seen, turn = np.zeros((3, hkv, 150)), np.zeros(3, int), [0]

    def arrays():
        c = {"k": kv.k, "v": kv.v, "k_scale": kv.k_scale, "v_scale": kv.v_scale, "table": kv.table}
        return {n: x.cpu().numpy().copy() for n, x in c.items() if x is not None}

    def step(new, depths=None, tree=None):
        turn[0] += 1
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        qkv = synth.normal(41, turn[0], (int(cu[-1]), (hq + 2 * hkv) * dh))
        before = arrays()
        kv.append(R.dev(qkv), new, depths)
        out = kv.attend(None if tree is None else R.dev(tree.view(np.int32))).cpu().numpy()
        pos = np.repeat(seen, new) + (np.concatenate([np.arange(n) for n in new]) if depths is None else np.asarray(depths))
        c = arrays()
        before["table"] = c["table"]
        K.append(before, qkv, hq, cu, kv.lens_host, pos, cos, sin)
        for n in c:
            assert same_bits(c[n], before[n]), n
        want, added, reach = K.attend(c, qkv, hq, cu, kv.lens_host, pos, cos, sin, tree)
        check_rows(out, want, reach, cu, len(qkv), 3)
        rw[:, :, :added.shape[2]] += added
        if depths is None:
            seen[:] += new
        assert np.array_equal(kv.lens.cpu().numpy(), kv.lens_host)

    step([100, 20, 0])
    step([1, 1, 1])
    step([30, 0, 2])                                                      # 131, 21 and 3 slots: 9, 2 and 1 pages
    with pytest.raises(MemoryError, match="no page left"):
        kv.append(torch.zeros(120, (hq + 2 * hkv) * dh, device="cuda"), [0, 120, 0])
    assert list(kv.lens_host) == [131, 21, 3] and list(kv.seen) == [131, 21, 3]
    lens, weights, was = kv.lens_host.copy(), kv.weights.cpu().numpy(), arrays()
    assert np.abs(weights - rw).max() <= 1e-5 * rw.max()
    kept = kv.evict(40, 2, 10).cpu().numpy()
    want, counts = K.select(weights, lens, 40, 2, 10)
    assert np.array_equal(kept, want) and list(kv.lens_host) == [40, 21, 3] and len(kv.free) == 17 - 3 - 2 - 1
    K.compact(was, lens, want, None, counts, rw)
    rw[0, :, 40:] = 0
    now = arrays()
    for n in now:
        if n != "table":
            assert same_bits(now[n], was[n]), n
    assert not kv.weights[0, :, 40:].any()
    step([1, 120, 3])                                                     # state 1 on the pages that state 0 gave up
    # three candidates of two tokens behind state 0, two of one behind state 2
    tree = np.array([1, 3, 4, 12, 16, 48, 1, 2], np.uint32)[:, None]
    step([6, 0, 2], [0, 1, 0, 1, 0, 1, 0, 0], tree)
    start = kv.lens_host - [6, 0, 2]
    before, lens = arrays(), kv.lens_host.copy()
    kv.keep_branch([[2, 3], [], [1]])
    branch = np.array([[[start[0] + 2, start[0] + 3]], [[-1, -1]], [[start[2] + 1, -1]]], np.int32)
    K.compact(before, lens, branch, start, [2, 0, 1], rw)
    now = arrays()
    for n in now:
        if n != "table":
            assert same_bits(now[n], before[n]), n
    seen[:] += [2, 0, 1]
    assert list(kv.seen) == list(seen) and np.array_equal(kv.lens_host, start + [2, 0, 1])
    for b in range(3):
        rw[b, :, kv.lens_host[b]:] = 0
    step([2, 1, 30])
    assert np.abs(kv.weights.cpu().numpy() - rw).max() <= 1e-5 * rw.max()


def test_the_holder_refuses():
    B, R = _mods()
    for bad in (dict(dtype=torch.bfloat16), dict(states=0), dict(head_dim=0), dict(max_tokens=0)):
        with pytest.raises(ValueError):
            R.KVCache(**{**dict(states=2, n_heads=4, n_kv_heads=2, head_dim=32, max_tokens=40, rope_theta=1e4, page_tokens=16), **bad})
    kv = R.KVCache(2, 4, 2, 32, 40, 1e4, page_tokens=16)
    rows = lambda n: torch.zeros(n, 8 * 32, device="cuda")  # noqa: E731
    for qkv, new, depths, word in ((rows(2), [1], None, "new"), (rows(2), [3, -1], None, "new"), (rows(0), [0, 0], None, "new"),
                                   (rows(3), [1, 1], None, "qkv"), (rows(2).half(), [1, 1], None, "qkv"), (rows(42), [41, 1], None, "max_tokens"),
                                   (rows(2), [1, 1], [0], "depths"), (rows(2), [1, 1], [0, -1], "depths"), (rows(2), [1, 1], [0, 40], "rotary")):
        with pytest.raises(ValueError, match=word):
            kv.append(qkv, new, depths)
    with pytest.raises(ValueError, match="append"):
        kv.attend()
    with pytest.raises(ValueError, match="append"):
        kv.keep_branch([[], []])
    with pytest.raises(ValueError, match="track_weights"):
        kv.evict(4, 0, 0)
    kv.append(rows(3), [2, 1])
    for bad in ([[0]], [[1, 0], []], [[0, 0], []], [[2], []], [[], [-1]]):
        with pytest.raises(ValueError, match="branch"):
            kv.keep_branch(bad)
    with pytest.raises(ValueError, match="tree_mask"):
        kv.attend(torch.zeros(2, 1, dtype=torch.int32, device="cuda"))
    kv.attend()
    kv.keep_branch([[1], [0]])
    with pytest.raises(ValueError, match="append"):
        kv.attend()


# ---------------------------------------------------------------- groups of every size, the same row several times

@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("dh,group,hkv,cached,new", [
    (32, 3, 2, [70, 5], [5, 4]), (64, 5, 1, [40], [3]), (64, 7, 2, [1100], [2]), (32, 16, 1, [90, 3], [1, 1]), (16, 17, 1, [64, 2], [1, 1]),
    (32, 48, 1, [33], [3]), (16, 6, 3, [3, 1500], [11, 2]),
])
def test_groups_of_every_size(dh, group, hkv, cached, new, dtype):
    B, R = _mods()
    print("group", dh, group, hkv, cached, new, dtype, flush=True)
    hq = group * hkv
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1])
    qkv = synth.normal(51, dh + group, (T, (hq + 2 * hkv) * dh))
    cos, sin = tables(max(lens), dh)
    c = make_cache(52, hkv, dh, 16, lens, DTYPES[dtype])
    w = torch.zeros(len(lens), hkv, max(lens), device="cuda")
    got = OnGpu(B, R, c, dh, cos, sin).attend(qkv, hq, cu, max(new), lens, weights=w)
    want, added, reach = K.attend(c, qkv, hq, cu, lens, None, cos, sin)
    check_rows(got, want, reach, cu, T, len(lens))
    g = w.cpu().numpy()
    assert np.all(np.abs(g - added) <= 4e-6 * added + 2.0 ** -23 * g)


@pytest.mark.parametrize("ld,shift", [(3001, 0), (3004, 1), (3004, 2), (3000, 0)])
def test_select_from_rows_on_any_four_bytes(ld, shift):
    """Rows of weights that do not start on 16 bytes, and the last row of memory that ends with the last slot."""
    B, R = _mods()
    w = np.abs(synth.normal(61, ld, (2, 3, ld)))
    flat = torch.zeros(w.size + 8, device="cuda")
    flat[shift:shift + w.size] = R.dev(w.ravel())
    t = flat[shift:shift + w.size].view(2, 3, ld)
    kept = torch.zeros(2, 3, 500, dtype=torch.int32, device="cuda")
    counts = torch.zeros(2, dtype=torch.int32, device="cuda")
    lens = np.array([3000, 2998], np.int32)
    B.attention_cache_select(t, 2, 3, R.dev(lens), 3000, 500, 3, 50, kept, counts)
    want, n = K.select(w, lens, 500, 3, 50)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), n)


# ---------------------------------------------------------------- the same call again

@pytest.mark.parametrize("dtype", ["f32", "f16", "i8"])
@pytest.mark.parametrize("dh,hq,hkv,page,cached,new", [
    (128, 8, 2, 64, [10, 300], [130, 77]),                        # shared blocks, weights in parts
    (64, 4, 2, 32, [1500, 3], [1, 2]),                            # the shared list
    (32, 6, 2, 16, [100, 40], [2, 1]),                            # a workgroup each
])
def test_captured_calls_with_weights_repeat_themselves(dh, hq, hkv, page, cached, new, dtype):
    """append, attention with weights, selection and moving in one graph: every replay gives the eager calls' bits.  In between the program
    works and synchronizes, and the cache, weights and workspace are put back or spoiled."""
    B, R = _mods()
    lens = [a + n for a, n in zip(cached, new)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, keep = int(cu[-1]), max(lens) // 2
    cos, sin = tables(max(lens), dh)
    c = make_cache(71, hkv, dh, page, lens, DTYPES[dtype])
    g = OnGpu(B, R, c, dh, cos, sin)
    start = {n: x.clone() for n, x in g.t.items()}
    qkv = R.dev(synth.normal(71, dh, (T, (hq + 2 * hkv) * dh)))
    cu_d, lens_d = g.ints(cu), g.ints(lens)
    w0 = torch.rand(len(lens), hkv, max(lens), device="cuda")
    w, out = w0.clone(), torch.empty(T, hq * dh, device="cuda")
    kept = torch.empty(len(lens), hkv, keep, dtype=torch.int32, device="cuda")
    counts = torch.empty(len(lens), dtype=torch.int32, device="cuda")
    ws = torch.empty(B.brl_attention_cached_workspace_bytes(g.struct, hq, T, len(lens), max(new), max(lens), True), dtype=torch.uint8, device="cuda")

    def calls():
        B.attention_cache_append(g.struct, qkv, hq, T, len(lens), cu_d, max(new), lens_d, None, g.cos, g.sin)
        B.attention_cached_forward(g.struct, qkv, hq, T, len(lens), cu_d, max(new), lens_d, max(lens), None, g.cos, g.sin, None, out, w, ws)
        B.attention_cache_select(w, len(lens), hkv, lens_d, max(lens), keep, 2, keep // 4, kept, counts)
        B.attention_cache_compact(g.struct, len(lens), lens_d, max(lens), kept, hkv, None, counts, w)

    def reset():
        for n, x in g.t.items():
            x.copy_(start[n])
        w.copy_(w0)
        ws.fill_(255)
        out.fill_(float("nan"))
        kept.fill_(-7)
        counts.fill_(-7)

    def state():
        torch.cuda.synchronize()
        return [x.cpu().numpy().copy() for x in (out, w, kept, counts, *g.t.values())]

    reset()
    calls()
    eager = state()
    reset()
    calls()
    assert all(same_bits(a, b) for a, b in zip(eager, state()))
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        reset()
        graph.replay()
        got = state()
        assert all(same_bits(a, b) for a, b in zip(eager, got))
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_two_streams_at_once():
    """Two calls in flight on two streams, each with its own cache, workspace and outputs, give what each gives alone."""
    B, R = _mods()
    dh, hq, hkv, page = 64, 4, 2, 32
    cos, sin = tables(3000, dh)
    jobs = []
    for i, (cached, new) in enumerate((([2500, 900], [2, 1]), ([400, 30], [90, 60]))):
        lens = [a + n for a, n in zip(cached, new)]
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        g = OnGpu(B, R, make_cache(81 + i, hkv, dh, page, lens, np.float16), dh, cos, sin)
        T = int(cu[-1])
        j = dict(g=g, T=T, new=max(new), longest=max(lens), qkv=R.dev(synth.normal(81, i, (T, (hq + 2 * hkv) * dh))), cu=g.ints(cu), lens=g.ints(lens),
                 stream=torch.cuda.Stream())
        j["ws"] = torch.empty(B.brl_attention_cached_workspace_bytes(g.struct, hq, T, 2, j["new"], j["longest"], True), dtype=torch.uint8, device="cuda")
        jobs.append(j)

    def run(j, out, w):
        B.attention_cached_forward(j["g"].struct, j["qkv"], hq, j["T"], 2, j["cu"], j["new"], j["lens"], j["longest"], None, j["g"].cos, j["g"].sin,
                                   None, out, w, j["ws"])

    def outputs(n):
        return [[(torch.empty(j["T"], hq * dh, device="cuda"), torch.zeros(2, hkv, j["longest"], device="cuda")) for _ in range(n)] for j in jobs]

    alone, together = outputs(1), outputs(20)
    for j, o in zip(jobs, alone):
        run(j, *o[0])
    torch.cuda.synchronize()
    for i in range(20):
        for j, o in zip(jobs, together):
            with torch.cuda.stream(j["stream"]):
                run(j, *o[i])
    torch.cuda.synchronize()
    for a, many in zip(alone, together):
        for o in many:
            assert torch.equal(o[0], a[0][0]) and torch.equal(o[1], a[0][1])
