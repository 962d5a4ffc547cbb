"""What chunk_attention, key_weights and evict_kv refuse, on the CPU: the binding by
tensor extents, the C entries by their arguments (their pointers are fake, and
every call fails a check)."""

import os

import pytest

from test_rows_and_attn_refusals import (EALIGN, EINVAL, EUNSUP, EWS, FAKE, LIB, F, I, P, S, Z, bf, bpc, call, expect, f32, i32, i64, lib, rows, z)

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libbpc.so not built")


# ------------------------------------------------------------- the binding
def chunk(bpc, **kw):
    a = dict(q=z(2, 8, 5, 128), K=z(2, 2, 32, 128), V=z(2, 2, 32, 128), pos=z(2, dtype=i32))
    a.update(kw)
    return bpc.chunk_attention(a.pop("q"), a.pop("K"), a.pop("V"), a.pop("pos"), **a)


def weigh(bpc, **kw):
    a = dict(q=z(2, 8, 5, 128), K=z(2, 2, 32, 128), lse=z(2, 8, 5, dtype=f32), weights=z(2, 2, 32, dtype=f32), pos=z(2, dtype=i32))
    a.update(kw)
    return bpc.key_weights(a.pop("q"), a.pop("K"), a.pop("lse"), a.pop("weights"), a.pop("pos"), **a)


def evict(bpc, **kw):
    a = dict(K=z(2, 2, 32, 128), V=z(2, 2, 32, 128), weights=z(2, 2, 32, dtype=f32), lens=z(2, dtype=i32), keep=20, K_out=z(2, 2, 20, 128),
             V_out=z(2, 2, 20, 128))
    a.update(kw)
    first = [a.pop(x) for x in ("K", "V", "weights", "lens", "keep", "K_out", "V_out")]
    return bpc.evict_kv(*first, **a)


TABLE = dict(K=z(7, 2, 16, 128), V=z(7, 2, 16, 128), block_table=z(2, 2, dtype=i32))
OUT_TABLE = dict(K_out=z(5, 2, 16, 128), V_out=z(5, 2, 16, 128), table_out=z(2, 2, dtype=i32))


def test_good_shapes_reach_the_device_check(bpc):
    expect(lambda: chunk(bpc, count=z(2, dtype=i32), slopes=z(8, dtype=f32), window=7, sinks=3, lse_out=z(2, 8, 5, dtype=f32)), "GPU")
    expect(lambda: chunk(bpc, N=20, **TABLE), "GPU")
    expect(lambda: chunk(bpc, window=2 ** 40, sinks=2 ** 40), "GPU")
    expect(lambda: weigh(bpc, count=z(2, dtype=i32), slopes=z(8, dtype=f32), weights=z(2, 2, 99, dtype=f32), decay=0.5), "GPU")
    expect(lambda: weigh(bpc, K=TABLE["K"], block_table=TABLE["block_table"], weights=z(2, 2, 30, dtype=f32)), "GPU")
    expect(lambda: evict(bpc, sinks=4, recent=16, codes=z(2, 2, 40, 2, dtype=i32), codes_out=z(2, 2, 20, 2, dtype=i32), weights_out=z(2, 2, 25, dtype=f32),
                         kept_out=z(2, 2, 20, dtype=i32)), "GPU")
    expect(lambda: evict(bpc, **TABLE, **OUT_TABLE), "GPU")


@pytest.mark.parametrize("kw,word", [
    (dict(q=z(2, 8, 5, 64)), "q"), (dict(q=z(2, 7, 5, 128)), "Hq"), (dict(K=z(3, 2, 32, 128)), "K"), (dict(V=z(2, 2, 31, 128)), "V"),
    (dict(V=z(2, 1, 32, 128)), "V"), (dict(N=33), "K"), (dict(N=0), "N"), (dict(pos=z(3, dtype=i32)), "pos"), (dict(pos=z(2, dtype=i64)), "pos"),
    (dict(count=z(1, dtype=i32)), "count"), (dict(window=-1), "window"), (dict(sinks=-1), "sinks"), (dict(slopes=z(2, dtype=f32)), "slopes"),
    (dict(lse_out=z(2, 8, 4, dtype=f32)), "lse_out"), (dict(lse_out=z(2, 8, 5)), "lse_out"), (dict(lse_out=z(1, 8, 5, dtype=f32).expand(2, 8, 5)), "overlap"),
    (dict(out=z(2, 8, 5, 128, dtype=f32)), "out"), (dict(out=z(1, 8, 5, 128).expand(2, 8, 5, 128)), "overlap"), (dict(workspace=z(9, dtype=f32)), "workspace"),
    (dict(TABLE, N=33), "block_table"), (dict(TABLE, block_table=z(1, 2, dtype=i32)), "block_table"), (dict(TABLE, K=z(7, 2, 24, 128), V=z(7, 2, 24, 128)), "power"),
    (dict(TABLE, V=z(8, 2, 16, 128)), "V"),
])
def test_chunk_refuses(bpc, kw, word):
    expect(lambda: chunk(bpc, **kw), word)


@pytest.mark.parametrize("kw,word", [
    (dict(q=z(2, 9, 5, 128)), "Hq"), (dict(K=z(2, 2, 32, 128, dtype=f32)), "K"), (dict(K=z(3, 2, 32, 128)), "K"), (dict(lse=z(2, 8, 6, dtype=f32)), "lse"),
    (dict(lse=z(2, 8, 5)), "lse"), (dict(weights=z(2, 3, 32, dtype=f32)), "weights"), (dict(weights=z(2, 2, 31, dtype=f32), N=32), "weights"),
    (dict(weights=z(2, 1, 32, dtype=f32).expand(2, 2, 32)), "overlap"), (dict(weights=z(2, 2, 64, dtype=f32)[..., ::2]), "weights"), (dict(pos=z(2, 1, dtype=i32)), "pos"),
    (dict(window=-2), "window"), (dict(K=TABLE["K"], block_table=TABLE["block_table"], N=33), "block_table"), (dict(slopes=z(9, dtype=f32)), "slopes"),
])
def test_weights_refuse(bpc, kw, word):
    expect(lambda: weigh(bpc, **kw), word)


@pytest.mark.parametrize("kw,word", [
    (dict(keep=0), "keep"), (dict(keep=33), "keep"), (dict(sinks=10, recent=11), "sinks"), (dict(sinks=-1), "sinks"), (dict(recent=-1), "recent"),
    (dict(lens=z(2, dtype=i64)), "lens"), (dict(lens=z(2, 1, dtype=i32)), "lens"), (dict(lens=z(3, dtype=i32)), "K"), (dict(V=z(2, 3, 32, 128)), "V"),
    (dict(K_out=z(2, 2, 19, 128)), "K_out"), (dict(V_out=z(2, 2, 19, 128)), "V_out"), (dict(K_out=z(1, 2, 20, 128).expand(2, 2, 20, 128)), "overlap"),
    (dict(weights=z(2, 2, 31, dtype=f32), N=32), "weights"), (dict(weights_out=z(2, 2, 19, dtype=f32)), "weights_out"), (dict(codes=z(2, 2, 32, 2, dtype=i32)), "codes"),
    (dict(codes=z(2, 2, 32, 3, dtype=i32), codes_out=z(2, 2, 20, 3, dtype=i32)), "codes"), (dict(kept_out=z(2, 2, 21, dtype=i32)), "kept_out"),
    (dict(codes=z(2, 2, 31, 2, dtype=i32), codes_out=z(2, 2, 20, 2, dtype=i32)), "codes"), (dict(codes=z(2, 2, 32, 2, dtype=i32), codes_out=z(2, 2, 20, 1, dtype=i32)), "codes_out"),
    (dict(OUT_TABLE, keep=32, table_out=z(2, 1, dtype=i32)), "table_out"), (dict(OUT_TABLE, V_out=z(4, 2, 16, 128)), "V_out"),
])
def test_evict_refuses(bpc, kw, word):
    expect(lambda: evict(bpc, **kw), word)


# ------------------------------------------------------------- the C entries
PAGES = [("table", P, FAKE), ("st", S, 400), ("pages", I, 900), ("page", I, 16)]
SIZES = [("B", I, 2), ("Hq", I, 8), ("Hkv", I, 2), ("T", I, 5), ("N", I, 5000), ("D", I, 128)]
SCORE = [("sm", F, 0.088), ("cap", F, 0.0), ("slopes", P, None), ("window", I, 0), ("sinks", I, 0)]
CHUNK = (rows("q", 8) + rows("K", 2) + rows("V", 2) + PAGES + [("pos", P, FAKE), ("count", P, None)] + SIZES + SCORE + rows("o", 8) +
         [("lse", P, None), ("lse_b", S, 40), ("lse_h", S, 5), ("ws", P, FAKE), ("wsb", Z, 1 << 40), ("stream", P, None)])
WEIGHTS = (rows("q", 8) + rows("K", 2) + [("lse", P, FAKE), ("lse_b", S, 40), ("lse_h", S, 5), ("w", P, FAKE), ("w_b", S, 10000), ("w_h", S, 5000)] + PAGES +
           [("pos", P, FAKE), ("count", P, None)] + SIZES + SCORE + [("decay", F, 1.0), ("stream", P, None)])
FAR = 1 << 40  # apart from FAKE by more than any span here
EVICT = ([("K", P, FAKE), ("K_b", S, 5000 * 256), ("K_h", S, 5000 * 128), ("K_t", S, 128), ("V", P, 2 * FAR), ("V_b", S, 5000 * 256), ("V_h", S, 5000 * 128), ("V_t", S, 128),
          ("table", P, None), ("st", S, 0), ("pages", I, 0), ("page", I, 0), ("w", P, 3 * FAR), ("w_b", S, 10000), ("w_h", S, 5000), ("lens", P, 4 * FAR), ("B", I, 2),
          ("Hkv", I, 2), ("N", I, 5000), ("D", I, 128), ("keep", I, 1000), ("sinks", I, 4), ("recent", I, 100),
          ("Ko", P, 5 * FAR), ("Ko_b", S, 1000 * 256), ("Ko_h", S, 1000 * 128), ("Ko_t", S, 128), ("Vo", P, 6 * FAR), ("Vo_b", S, 1000 * 256), ("Vo_h", S, 1000 * 128),
          ("Vo_t", S, 128), ("to", P, None), ("sto", S, 0), ("opages", I, 0), ("opage", I, 0), ("codes", P, None), ("C_b", S, 20000), ("C_h", S, 10000), ("co", P, None),
          ("Co_b", S, 4000), ("Co_h", S, 2000), ("W", I, 2), ("wo", P, None), ("wo_b", S, 2000), ("wo_h", S, 1000), ("cap", I, 1000), ("kept", P, 7 * FAR), ("ws", P, None),
          ("wsb", Z, 0), ("stream", P, None)])

ANY = [
    (dict(q=None), EINVAL), (dict(K=None), EINVAL), (dict(B=0), EINVAL), (dict(T=0), EINVAL), (dict(N=0), EINVAL), (dict(Hq=9), EINVAL), (dict(Hq=2 * 129), EUNSUP),
    (dict(D=64), EUNSUP), (dict(sm=0.0), EINVAL), (dict(sm=float("nan")), EINVAL), (dict(cap=-1.0), EINVAL), (dict(cap=1025.0), EUNSUP), (dict(cap=2.0 ** -21), EUNSUP),
    (dict(sm=2.0 ** -41), EUNSUP), (dict(sm=2.0 ** 41), EUNSUP), (dict(slopes=FAKE + 2), EALIGN), (dict(q=FAKE + 2), EALIGN), (dict(K_t=100), EINVAL), (dict(K_t=132), EALIGN),
    (dict(K_t=1 << 25), EUNSUP), (dict(q_h=-8), EINVAL), (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(pos=None), EINVAL), (dict(pos=FAKE + 2), EALIGN),
    (dict(count=FAKE + 1), EALIGN), (dict(page=17), EINVAL), (dict(page=1 << 21), EINVAL), (dict(pages=0), EINVAL), (dict(st=-1), EINVAL), (dict(table=FAKE + 2), EALIGN),
    (dict(B=1 << 20), EUNSUP),
]


@pytest.mark.parametrize("kw,code", ANY + [
    (dict(V=None), EINVAL), (dict(o=None), EINVAL), (dict(o=FAKE + 8), EALIGN), (dict(o_h=64), EINVAL), (dict(o_t=64), EINVAL), (dict(V_t=1 << 25), EUNSUP),
    (dict(ws=None), EWS), (dict(wsb=256), EWS), (dict(ws=FAKE + 16), EALIGN), (dict(lse=FAKE + 2), EALIGN), (dict(lse=FAKE, lse_h=4), EINVAL),
    (dict(lse=FAKE, lse_b=-1), EINVAL), (dict(lse=FAKE, lse_b=39), EINVAL), (dict(T=1 << 30), EUNSUP),
])
def test_chunk_entry_rejects(lib, kw, code):
    assert call(lib, "bpc_chunk_attention", CHUNK, kw) == code
    assert lib.bpc_last_error() != b""


@pytest.mark.parametrize("kw,code", ANY + [
    (dict(lse=None), EINVAL), (dict(lse=FAKE + 2), EALIGN), (dict(lse_h=-1), EINVAL), (dict(w=None), EINVAL), (dict(w=FAKE + 1), EALIGN), (dict(w_h=4999), EINVAL),
    (dict(w_b=9999), EINVAL), (dict(decay=-0.5), EINVAL), (dict(decay=float("inf")), EINVAL), (dict(decay=float("nan")), EINVAL),
])
def test_weights_entry_rejects(lib, kw, code):
    assert call(lib, "bpc_key_weights", WEIGHTS, kw) == code
    assert lib.bpc_last_error() != b""


CODES = dict(codes=8 * FAR, co=9 * FAR)
PAGED = dict(table=FAKE, st=400, pages=900, page=16, to=FAKE, sto=70, opages=900, opage=16, K_b=4096, K_h=2048, V_b=4096, V_h=2048, Ko_b=4096, Ko_h=2048, Vo_b=4096, Vo_h=2048)


@pytest.mark.parametrize("kw,code", [
    (dict(K=None), EINVAL), (dict(V=None), EINVAL), (dict(w=None), EINVAL), (dict(lens=None), EINVAL), (dict(kept=None), EINVAL), (dict(Ko=None), EINVAL),
    (dict(Vo=None), EINVAL), (dict(B=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(N=0), EINVAL), (dict(D=64), EUNSUP), (dict(keep=0), EINVAL), (dict(keep=5001), EINVAL),
    (dict(sinks=901), EINVAL), (dict(sinks=-1), EINVAL), (dict(recent=-1), EINVAL), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), EINVAL), (dict(K=FAKE + 8), EALIGN),
    (dict(Ko_t=64), EINVAL), (dict(Vo_h=0), EINVAL), (dict(Ko_t=132), EALIGN), (dict(w=3 * FAR + 2), EALIGN), (dict(w_b=-1), EINVAL), (dict(kept=7 * FAR + 2), EALIGN),
    (dict(Ko=FAKE + 256), EINVAL), (dict(Vo=FAKE + 256 * 5000), EINVAL), (dict(Ko=6 * FAR), EINVAL), (dict(codes=8 * FAR), EINVAL), (dict(co=8 * FAR), EINVAL),
    (dict(CODES, W=3), EUNSUP), (dict(CODES, codes=8 * FAR + 4), EALIGN), (dict(CODES, Co_h=1999), EALIGN), (dict(CODES, Co_h=1998), EINVAL), (dict(CODES, co=8 * FAR + 160), EINVAL),
    (dict(wo=8 * FAR, cap=999), EINVAL), (dict(wo=8 * FAR, wo_h=999), EINVAL), (dict(wo=3 * FAR + 400), EINVAL), (dict(wo=7 * FAR), EINVAL), (dict(kept=3 * FAR), EINVAL),
    (dict(kept=4 * FAR), EINVAL), (dict(PAGED, page=24), EINVAL), (dict(PAGED, opage=8), EINVAL), (dict(PAGED, pages=0), EINVAL), (dict(PAGED, opages=0), EINVAL),
    (dict(PAGED, sto=-1), EINVAL), (dict(PAGED, Vo=5 * FAR), EINVAL), (dict(PAGED, N=50000), EWS), (dict(N=50000, K_h=50000 * 128, K_b=10 ** 8, V_h=50000 * 128, V_b=10 ** 8, w_h=50000, w_b=10 ** 5), EWS),
    (dict(PAGED, N=50000, ws=FAKE + 16, wsb=1 << 40), EALIGN), (dict(B=1 << 20), EUNSUP),
])
def test_evict_entry_rejects(lib, kw, code):
    assert call(lib, "bpc_evict_kv", EVICT, kw) == code
    assert lib.bpc_last_error() != b""


@pytest.mark.parametrize("kw", [dict(Ko=FAKE + 4000 * 256), dict(Ko=FAKE + 4000 * 256, Vo=2 * FAR + 4000 * 256), dict(Vo=FAKE + 4000 * 256)])
def test_evict_takes_other_rows_of_one_buffer(lib, kw):
    """Rows behind those that are read, in buffers of 5000 rows a head, are apart from them."""
    strides = dict(Ko_b=5000 * 256, Ko_h=5000 * 128, Vo_b=5000 * 256, Vo_h=5000 * 128)
    assert call(lib, "bpc_evict_kv", EVICT, dict(strides, N=4000, kept=None, **kw)) == EINVAL and b"kept" in lib.bpc_last_error()
    assert call(lib, "bpc_evict_kv", EVICT, dict(strides, N=4001, kept=None, **kw)) == EINVAL and b"overlaps" in lib.bpc_last_error()


def test_sizes(lib):
    import ctypes
    for name in ("bpc_chunk_workspace_bytes", "bpc_evict_workspace_bytes"):
        getattr(lib, name).restype = ctypes.c_size_t
    ws = lib.bpc_chunk_workspace_bytes
    assert ws(1, 32, 8, 1, 16384, 128, 0, 0) > ws(1, 32, 8, 1, 16384, 128, 1024, 4) > 0
    assert ws(1, 32, 8, 1, 16384, 128, 0, 0) % 256 == 0
    assert ws(1, 32, 8, 1, 100, 128, 0, 0) == 0  # one step
    assert ws(1, 32, 8, 1, 16384, 64, 0, 0) == ws(1, 30, 8, 1, 16384, 128, 0, 0) == ws(1, 32, 8, 1, 16384, 128, -1, 0) == 0
    assert ws(1, 32, 8, 1, 16384, 128, 2 ** 31 - 1, 2 ** 31 - 1) == ws(1, 32, 8, 1, 16384, 128, 1 << 30, 1 << 30)
    ev = lib.bpc_evict_workspace_bytes
    assert ev(2, 8, 16384, 100) == 0 and ev(2, 8, 16385, 100) > 0 and ev(2, 8, 16385, 100) % 4 == 0
    assert ev(0, 8, 20000, 5) == ev(2, 8, 20000, 0) == ev(2, 8, 20000, 20001) == 0


@pytest.mark.parametrize("kw,word", [
    (dict(Vo=5 * FAR + 256, Vo_t=256, Vo_h=2000 * 256, Vo_b=4000 * 256), b"overlaps"), (dict(w_b=(1 << 40) + 1), b"2^40"), (dict(wo=8 * FAR, wo_h=1 << 41), b"2^40"),
    (dict(CODES, C_b=1 << 41), b"2^40"),
])
def test_evict_entry_says_why(lib, kw, word):
    """Results at other strides within one another's reach, and strides that no memory has."""
    assert call(lib, "bpc_evict_kv", EVICT, kw) == EINVAL
    assert word in lib.bpc_last_error()
