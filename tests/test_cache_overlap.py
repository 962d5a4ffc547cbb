"""What chunk_attention, key_weights and evict_kv write shares no memory with anything
else, on the CPU (fake pointers; every call fails a check)."""

import random

import pytest

from test_cache_refusals import CHUNK, CODES, EVICT, WEIGHTS
from test_rows_and_attn_refusals import EINVAL, call, lib, pytestmark  # noqa: F401

FAR = 1 << 40  # further than any argument here reaches
SIZES = dict(B=2, Hq=8, Hkv=2, T=5, N=5000)
LSE = 2 * 8 * 5 * 4  # bytes


def apart(names):
    return {name: (i + 1) * FAR for i, name in enumerate(names)}


# q, out [2, 8, 5, 128], K, V [2, 2, 5000, 128]
Q, KV = dict(b=5120, h=640, t=128), dict(b=1280000, h=640000, t=128)
DENSE = dict({"q_" + k: v for k, v in Q.items()}, **{"o_" + k: v for k, v in Q.items()}, **{"K_" + k: v for k, v in KV.items()}, **{"V_" + k: v for k, v in KV.items()})
CHUNK_GOOD = dict(SIZES, **DENSE, **apart(["q", "K", "V", "pos", "count", "slopes", "o", "lse", "ws"]), table=None, lse_b=40, lse_h=5)
POOL = dict(table=20 * FAR, st=400, pages=900, page=16, K_b=4096, K_h=2048, V_b=4096, V_h=2048)


def refused(lib, entry, spec, kw, *words):
    assert call(lib, entry, spec, kw) == EINVAL, kw
    said = lib.bpc_last_error().decode()
    assert "overlaps" in said and all(w in said for w in words), said


# an argument, and the bytes it covers
READ = [("q", 20480), ("K", 5120000), ("V", 5120000), ("pos", 8), ("count", 8), ("slopes", 32)]


@pytest.mark.parametrize("written,size", [("o", 20480), ("lse", LSE)])
@pytest.mark.parametrize("name,bytes", READ)
def test_chunk_refuses_results_on_its_inputs(lib, written, size, name, bytes):
    good = CHUNK_GOOD
    for at in (good[name], good[name] + bytes - 4 if written == "lse" else good[name] + (bytes - 1) // 16 * 16, good[name] - (size - 16)):
        refused(lib, "bpc_chunk_attention", CHUNK, dict(good, **{written: at}), "out" if written == "o" else "lse", name)


@pytest.mark.parametrize("written", ["o", "lse"])
def test_chunk_refuses_results_on_pools_and_tables(lib, written):
    good = dict(CHUNK_GOOD, **POOL)
    for name, at in (("K", good["K"] + 900 * 8192 - 16), ("V", good["V"]), ("block_table", good["table"] + 4 * (400 + 312))):
        refused(lib, "bpc_chunk_attention", CHUNK, dict(good, **{written: at}), name)


def test_chunk_refuses_results_on_one_another(lib):
    refused(lib, "bpc_chunk_attention", CHUNK, dict(CHUNK_GOOD, lse=CHUNK_GOOD["o"] + 20476), "out", "lse")
    refused(lib, "bpc_chunk_attention", CHUNK, dict(CHUNK_GOOD, T=1, ws=CHUNK_GOOD["o"] - 256), "out", "workspace")
    refused(lib, "bpc_chunk_attention", CHUNK, dict(CHUNK_GOOD, T=1, ws=CHUNK_GOOD["lse"]), "lse", "workspace")
    refused(lib, "bpc_chunk_attention", CHUNK, dict(CHUNK_GOOD, T=1, ws=CHUNK_GOOD["K"]), "workspace", "K")


def told(lib, out, lse):
    """Whether out and lse are found to overlap; where not, the call fails at the workspace, which comes later."""
    kw = dict(CHUNK_GOOD, **out, **lse)
    kw["ws"] = kw["q"]
    assert call(lib, "bpc_chunk_attention", CHUNK, kw) == EINVAL
    said = lib.bpc_last_error().decode()
    assert said in ("out overlaps lse", "workspace overlaps q"), said
    return said == "out overlaps lse"


def test_chunk_takes_results_that_lie_between_one_another(lib):
    """A sequence's rows and its log-sums behind them, in one buffer."""
    out = dict(o=30 * FAR, o_b=5200, o_h=640, o_t=128)
    assert not told(lib, out, dict(lse=30 * FAR + 10240, lse_b=2600, lse_h=5))
    assert told(lib, out, dict(lse=30 * FAR + 10236, lse_b=2600, lse_h=5))
    assert told(lib, out, dict(lse=30 * FAR + 10244, lse_b=2600, lse_h=5))
    assert told(lib, out, dict(lse=30 * FAR + 10240, lse_b=2598, lse_h=5))


def test_chunk_results_in_any_layout(lib):
    """Against the bytes themselves: views of one buffer, in any order of the dimensions, padded and not."""
    rng = random.Random(1)
    B, H, T = SIZES["B"], SIZES["Hq"], SIZES["T"]
    met = 0
    for case in range(400):
        def layout(dims, unit, span):
            stride = {}
            for name, n in rng.sample(dims, len(dims)):
                stride[name] = (span + rng.choice([0, 0, unit, 40 * unit, 2 * span, 16 * span]) + unit - 1) // unit * unit
                span = stride[name] * (n - 1) + span
            return stride
        o = layout([("b", B), ("h", H), ("t", T)], 16, 256)
        s = layout([("b", B), ("h", H)], 4, 4 * T)
        if rng.random() < 0.4:  # of one stride, as views of one buffer are
            s["b"], s["h"] = (max(o["b"], 4 * T * H), max(o["h"], 4 * T))
            s["b"] = max(s["b"], s["h"] * (H - 1) + 4 * T) if s["b"] >= s["h"] else s["b"]
        rows = [i * o["b"] + j * o["h"] + k * o["t"] for i in range(B) for j in range(H) for k in range(T)]
        sums = [i * s["b"] + j * s["h"] for i in range(B) for j in range(H)]
        row, one = rng.choice(rows), rng.choice(sums)
        away = rng.choice([0, 256, row + 256 - one, row + 256 - one, row - 4 * T - one, row - 4 * T - one, row + 4 * rng.randrange(64) - one, 4 * rng.randrange(-99, 99)])
        taken = {r + i for r in rows for i in range(0, 256, 4)}
        want = any(away + x + 4 * i in taken for x in sums for i in range(T))
        got = told(lib, dict(o=30 * FAR, o_b=o["b"] // 2, o_h=o["h"] // 2, o_t=o["t"] // 2), dict(lse=30 * FAR + away, lse_b=s["b"] // 4, lse_h=s["h"] // 4))
        assert got == want, (case, o, s, away)
        met += want
    assert 100 < met < 350, met


WEIGHTS_GOOD = dict(SIZES, **{k: v for k, v in DENSE.items() if k[:2] in ("q_", "K_")}, **apart(["q", "K", "pos", "count", "slopes", "lse", "w"]), table=None,
                    lse_b=40, lse_h=5, w_b=10000, w_h=5000)


@pytest.mark.parametrize("name,bytes", [("q", 20480), ("K", 5120000), ("pos", 8), ("count", 8), ("slopes", 32), ("lse", LSE)])
def test_weights_refuse_inputs(lib, name, bytes):
    for at in (WEIGHTS_GOOD[name], WEIGHTS_GOOD[name] + bytes - 4, WEIGHTS_GOOD[name] - 79996):
        refused(lib, "bpc_key_weights", WEIGHTS, dict(WEIGHTS_GOOD, w=at), "weights", name)


def test_weights_refuse_pools_and_tables(lib):
    pool = {k: v for k, v in POOL.items() if k[0] != "V"}
    for name, at in (("K", WEIGHTS_GOOD["K"] + 900 * 8192 - 16), ("block_table", pool["table"] + 4 * (400 + 312))):
        refused(lib, "bpc_key_weights", WEIGHTS, dict(WEIGHTS_GOOD, **pool, w=at), "weights", name)


def test_weights_take_what_lies_between(lib):
    """The log-sums of a head behind its weights, in one buffer; the call then fails at the lengths."""
    at = WEIGHTS_GOOD["w"]
    spaced = dict(WEIGHTS_GOOD, B=1, Hq=2, w_h=5008, lse_h=5008, pos=at + 4 * 4999)
    refused(lib, "bpc_key_weights", WEIGHTS, dict(spaced, lse=at + 4 * 5000), "weights", "pos")
    refused(lib, "bpc_key_weights", WEIGHTS, dict(spaced, lse=at + 4 * 4999), "weights", "lse")
    refused(lib, "bpc_key_weights", WEIGHTS, dict(spaced, lse=at + 4 * 5004), "weights", "lse")


# K, V, weights, lens, K_out, V_out, kept, codes, codes_out at 0, 2, 3 .. 9 (EVICT's own), then:
EVICT_GOOD = dict(CODES, K=FAR, wo=10 * FAR, to=11 * FAR, sto=70, opages=900, opage=16, Ko_b=4096, Ko_h=2048, Vo_b=4096, Vo_h=2048)
AT = dict(K=FAR, V=2 * FAR, weights=3 * FAR, lens=4 * FAR, K_out=5 * FAR, V_out=6 * FAR, kept=7 * FAR, codes=8 * FAR,
          table_out=11 * FAR)
POOLS = dict(POOL, K=FAR)


@pytest.mark.parametrize("result,word", [("Ko", "K_out"), ("Vo", "V_out")])
@pytest.mark.parametrize("name,bytes", [("weights", 80000), ("lens", 8), ("codes", 160000), ("table_out", 4 * (70 + 63))])
def test_evict_refuses_rows_on_its_inputs(lib, result, word, name, bytes):
    for at in (AT[name], AT[name] + (bytes - 1) // 16 * 16, AT[name] - 900 * 8192 + 16):
        refused(lib, "bpc_evict_kv", EVICT, dict(EVICT_GOOD, **{result: at}), word, name)
    refused(lib, "bpc_evict_kv", EVICT, dict(EVICT_GOOD, **dict(POOLS, table=AT["K_out"] + 900 * 8192 - 4)), "K_out", "block_table")


@pytest.mark.parametrize("result,word", [("wo", "weights_out"), ("co", "codes_out"), ("kept", "kept")])
@pytest.mark.parametrize("name,bytes", [("K", 5120000), ("V", 5120000), ("K_out", 900 * 8192), ("V_out", 900 * 8192), ("table_out", 4 * (70 + 63))])
def test_evict_refuses_results_on_rows_and_tables(lib, result, word, name, bytes):
    for at in (AT[name], AT[name] + (bytes - 1) // 16 * 16):
        refused(lib, "bpc_evict_kv", EVICT, dict(EVICT_GOOD, **{result: at}), word, name)


def test_evict_refuses_a_workspace_on_anything(lib):
    need = dict(EVICT_GOOD, N=50000, K_h=50000 * 128, K_b=10 ** 8, V_h=50000 * 128, V_b=10 ** 8, w_h=50000, w_b=10 ** 5, C_h=10 ** 5, C_b=2 * 10 ** 5, wsb=1 << 40)
    for name, at in AT.items():
        refused(lib, "bpc_evict_kv", EVICT, dict(need, ws=at), name, "workspace")
