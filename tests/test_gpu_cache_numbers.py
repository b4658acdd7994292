"""GPU tests of what numbers the key/value cache and its attention carry: new rows that are no numbers."""
import numpy as np
import pytest

from oracle import cache_oracle as K
from paper_2604_24273_amd import synth
from test_gpu_cache import OnGpu, _mods, make_cache, same_bits, tables

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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
