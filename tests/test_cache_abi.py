"""Host-side checks of the key/value cache entry points that need no GPU: sizes, refusals before any launch, marshalling."""
import ctypes as C
import os

import pytest

FAKE, ODD = 0x1000, 0x1004          # aligned and not, never dereferenced: checks fail first


@pytest.fixture(scope="module")
def B():
    from paper_2604_24273_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_24273_amd import build
        build.build()
    binding.lib()
    return binding


def cache(B, **kw):
    f = dict(n_pages=8, page_tokens=32, n_kv_heads=2, head_dim=64, dtype=B.BRL_F16, table_pages=4, k=FAKE, v=FAKE, k_scale=None,
             v_scale=None, page_table=FAKE)
    f.update(kw)
    return B.brl_kv_cache(*[f[n] for n, _ in B.brl_kv_cache._fields_])


def test_sizes(B):
    assert B.brl_kv_page_bytes(32, 5, 128, B.BRL_F16) == 32 * 5 * 128 * 2
    assert B.brl_kv_page_bytes(16, 4, 100, B.BRL_F32) == 16 * 4 * 112 * 4      # rows of 100 take 112 elements
    assert B.brl_kv_page_bytes(256, 1, 16, B.BRL_I8) == 256 * 16
    for bad in ((8, 1, 64, 0), (48, 1, 64, 0), (512, 1, 64, 0), (32, 0, 64, 0), (32, 1, 80, 0), (32, 1, 64, 1), (32, 1, 64, 9)):
        assert B.brl_kv_page_bytes(*bad) == 0
    assert C.sizeof(B.brl_kv_cache) == 6 * 4 + 5 * C.sizeof(C.c_void_p)
    need = lambda *a: B.brl_attention_cached_workspace_bytes(cache(B), *a)  # noqa: E731
    assert need(4, 8, 8, 1, 128, True) > 0
    for bad in ((3, 8, 8, 1, 128), (4, 0, 8, 1, 128), (4, 8, 0, 1, 128), (4, 8, 8, 0, 128), (4, 8, 8, 1, 0)):
        assert need(*bad, False) == 0
    assert need(4, 8, 8, 9, 128, True) == need(4, 8, 8, 8, 128, True)             # a bound past the tokens of the call
    assert B.brl_attention_cached_workspace_bytes(cache(B, head_dim=80), 4, 8, 8, 1, 128, False) == 0


def test_caches_are_checked(B):
    lib = B.lib()
    err = lambda: lib.brl_last_error().decode()  # noqa: E731

    def append(c, hq=4, T=8, states=8, cu=None, max_new=1, qkv=FAKE, lens=FAKE, cos=FAKE, sin=FAKE, rope=16):
        return lib.attention_cache_append(None if c is None else C.byref(c), qkv, hq, T, states, cu, max_new, lens, None, cos, sin, rope, None)

    assert append(None) == B.BRL_EINVAL and "null cache" in err()
    for bad, word in ((dict(page_tokens=24), "page_tokens"), (dict(page_tokens=8), "page_tokens"), (dict(page_tokens=512), "page_tokens"),
                      (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=96), "head_dim"), (dict(dtype=B.BRL_BF16), "dtype"),
                      (dict(n_pages=0), "n_pages"), (dict(table_pages=0), "table_pages"), (dict(table_pages=1 << 30), "table_pages"),
                      (dict(n_pages=2 ** 25), "rows"), (dict(k=None), "null"), (dict(v=ODD), "misaligned"), (dict(page_table=None), "null"),
                      (dict(dtype=B.BRL_I8), "k_scale"), (dict(k_scale=FAKE), "k_scale"),
                      (dict(dtype=B.BRL_I8, k_scale=FAKE), "v_scale"), (dict(dtype=B.BRL_I8, k_scale=ODD, v_scale=FAKE), "k_scale"),
                      (dict(dtype=B.BRL_I8, k_scale=FAKE, v_scale=ODD), "v_scale")):
        assert append(cache(B, **bad)) == B.BRL_EINVAL and word in err(), bad
    ok = cache(B)
    for bad, word in ((dict(hq=3), "n_heads"), (dict(hq=0), "n_heads"), (dict(T=0), "T = 0"), (dict(states=0), "B = 0"), (dict(max_new=0), "max_new"),
                      (dict(max_new=9), "max_new"), (dict(max_new=2), "T / B"), (dict(T=9), "T / B"), (dict(rope=0), "rope_len"),
                      (dict(qkv=None), "null"), (dict(qkv=ODD), "misaligned"), (dict(lens=None), "null"), (dict(cos=None), "null"),
                      (dict(sin=ODD), "misaligned"), (dict(T=1 << 29, cu=FAKE), "T ="), (dict(T=1 << 28, states=64, cu=FAKE, max_new=1 << 26), "too much")):
        assert append(ok, **bad) == B.BRL_EINVAL and word in err(), (bad, err())


def test_attention_select_and_compact_arguments(B):
    lib = B.lib()
    err = lambda: lib.brl_last_error().decode()  # noqa: E731
    ok = cache(B)

    def attend(out=FAKE, max_len=128, tree=None, words=0, weights=None, ldw=0, ws=FAKE, nbytes=1 << 40):
        return lib.attention_cached_forward(C.byref(ok), FAKE, 4, 8, 8, None, 1, FAKE, max_len, None, FAKE, FAKE, 16, tree, words, out,
                                            weights, ldw, ws, nbytes, None)

    for bad, word in ((dict(out=None), "null"), (dict(out=ODD), "misaligned"), (dict(ws=None), "null"), (dict(max_len=0), "max_len"),
                      (dict(max_len=129), "max_len"), (dict(tree=FAKE), "mask_words"), (dict(words=1), "mask_words"),
                      (dict(tree=FAKE, words=-1), "mask_words"), (dict(weights=FAKE, ldw=127), "ld_weights")):
        assert attend(**bad) == B.BRL_EINVAL and word in err(), (bad, err())
    assert attend(nbytes=0) == B.BRL_ENOSPC and "workspace" in err()

    def select(w=FAKE, ldw=100, states=2, hkv=2, lens=FAKE, max_len=100, keep=10, first=2, recent=3, kept=FAKE, counts=FAKE):
        return lib.attention_cache_select(w, ldw, states, hkv, lens, max_len, keep, first, recent, kept, counts, None)

    for bad, word in ((dict(w=None), "null"), (dict(lens=None), "null"), (dict(kept=None), "null"), (dict(counts=None), "null"),
                      (dict(states=0), "B = 0"), (dict(hkv=0), "n_kv_heads"), (dict(max_len=0), "max_len"), (dict(ldw=99), "ld_weights"),
                      (dict(keep=0), "keep"), (dict(first=-1), "first"), (dict(recent=-1), "recent"), (dict(first=8), "keep"),
                      (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), "keep"), (dict(states=1 << 22), "B =")):
        assert select(**bad) == B.BRL_EINVAL and word in err(), (bad, err())

    def compact(states=2, lens=FAKE, max_len=100, kept=FAKE, heads=1, ld=10, counts=FAKE, weights=None, ldw=0):
        return lib.attention_cache_compact(C.byref(ok), states, lens, max_len, kept, heads, ld, None, counts, weights, ldw, None)

    for bad, word in ((dict(lens=None), "null"), (dict(kept=None), "null"), (dict(counts=None), "null"), (dict(states=0), "B = 0"),
                      (dict(max_len=129), "max_len"), (dict(heads=3), "kept_heads"), (dict(heads=0), "kept_heads"), (dict(ld=0), "ld_kept"),
                      (dict(weights=FAKE, ldw=99), "ld_weights"), (dict(states=1 << 20), "B =")):
        assert compact(**bad) == B.BRL_EINVAL and word in err(), (bad, err())

    def rope(cos=FAKE, sin=FAKE, n=16, dh=64, theta=1e4):
        return lib.attention_rope_table(cos, sin, n, dh, theta, None)

    for bad in (dict(cos=None), dict(sin=ODD), dict(n=0), dict(dh=7), dict(dh=0), dict(dh=256), dict(theta=0.0), dict(n=1 << 25)):
        assert rope(**bad) == B.BRL_EINVAL, bad


def test_struct_builder_checks_tensors(B):
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 32, 112, dtype=torch.float16)
    table = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="rows of a cache"):
        B.make_kv_cache(k, k, None, None, table, 128)
    with pytest.raises(ValueError, match="one shape"):
        B.make_kv_cache(k, k.float(), None, None, table, 100)
    with pytest.raises(ValueError, match="one shape"):
        B.make_kv_cache(k.bfloat16(), k.bfloat16(), None, None, table, 100)
    with pytest.raises(ValueError, match="scales"):
        B.make_kv_cache(k.to(torch.int8), k.to(torch.int8), torch.zeros(4, 2, 31), torch.zeros(4, 2, 32), table, 100)
    with pytest.raises(ValueError, match="page_table"):
        B.make_kv_cache(k, k, None, None, table.long(), 100)
    with pytest.raises(ValueError, match="GPU"):
        B.make_kv_cache(k, k, None, None, table, 100)


def test_what_is_too_much_for_one_call(B):
    lib = B.lib()
    err = lambda: lib.brl_last_error().decode()  # noqa: E731
    large = cache(B, n_kv_heads=1, table_pages=1 << 20)

    def attend(hq, T, states, max_new, max_len=64, weights=None):
        rc = lib.attention_cached_forward(C.byref(large), FAKE, hq, T, states, FAKE, max_new, FAKE, max_len, None, FAKE, FAKE, 16, None, 0,
                                          FAKE, weights, max_len if weights else 0, FAKE, 0, None)
        return rc, B.brl_attention_cached_workspace_bytes(large, hq, T, states, max_new, max_len, weights is not None)

    # a workspace of 0 bytes is refused behind everything else
    rc, need = attend(4096, 255, 1, 255)
    assert rc == B.BRL_ENOSPC and need > 0
    for call in ((4096, 256, 1, 256),                               # 256 tokens x 4096^2
                 (4, 1 << 25, 1, 1 << 25), (4096, 1025, 1025, 1), (1, 1 << 23, 1 << 23, 1)):
        rc, need = attend(*call)
        assert rc == B.BRL_EINVAL and "too much" in err() and need == 0, call
    rc, need = attend(1, 64, 64, 1, 1 << 24, FAKE)
    assert rc == B.BRL_ENOSPC and need > 0
    rc, need = attend(1, 65, 65, 1, 1 << 24, FAKE)
    assert rc == B.BRL_EINVAL and "too many weights" in err() and need == 0
