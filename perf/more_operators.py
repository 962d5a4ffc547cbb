"""Timed cases of the operators that keep a cache small: attention of new tokens
over a paged cache, with a sliding window and first slots that stay visible
(``chunk_attention``), the attention weight that each cached slot gathers
(``key_weights``), and the eviction of the slots that gather the least
(``evict_kv``), with their plain forms in torch.

Head dim is 128 throughout, rows are bf16, weights fp32.  With ``own`` set,
``run`` makes the framework's calls; otherwise it computes the same in elementary
torch operations in 32 bits, rounded once at the end.  ``exact`` is the definition
in 64 bits.
"""

import math

import torch

own = False

D = 128
DEV = "cuda"


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one token of one request behind a window: launch latency
        dict(name="chunk_step_b1_window", kind="chunk", B=1, Hq=32, Hkv=8, T=1, N=16384, page=16, window=4096, sinks=4, cap=0.0, alibi=False, lse=False),
        # a batch's step at long context that reads a quarter of the cache
        dict(name="chunk_step_b16_64k_window", kind="chunk", B=16, Hq=32, Hkv=8, T=1, N=65536, page=64, window=16384, sinks=64, cap=0.0, alibi=False, lse=False),
        # short ragged prompts, log-sum-exp kept for the weights
        dict(name="chunk_b3_257", kind="chunk", B=3, Hq=32, Hkv=8, T=257, N=300, page=16, window=0, sinks=0, cap=0.0, alibi=False, lse=True),
        # prefill chunks of two requests over what is cached of them
        dict(name="chunk_b2_2048_32k", kind="chunk", B=2, Hq=32, Hkv=8, T=2048, N=32768, page=64, window=0, sinks=0, cap=0.0, alibi=False, lse=True),
        # a long prompt of odd length under a window
        dict(name="chunk_8001_window", kind="chunk", B=1, Hq=32, Hkv=8, T=8001, N=8192, page=128, window=1024, sinks=16, cap=0.0, alibi=False, lse=False),
        # capped scores with a distance bias, contiguous cache
        dict(name="chunk_b2_1000_16k_cap_bias", kind="chunk", B=2, Hq=32, Hkv=8, T=1000, N=16384, page=0, window=0, sinks=0, cap=50.0, alibi=True, lse=False),
        # what one token adds to a short cache: launch latency
        dict(name="weights_step_b1_4k", kind="weights", B=1, Hq=32, Hkv=8, T=1, N=4096, page=16, window=0, sinks=0, cap=0.0, alibi=False, decay=1.0),
        # what a batch's tokens add at long context, older weights fading
        dict(name="weights_step_b16_64k", kind="weights", B=16, Hq=32, Hkv=8, T=1, N=65536, page=64, window=0, sinks=0, cap=0.0, alibi=False, decay=0.98),
        # what the last tokens of two prompts look at
        dict(name="weights_b2_500_32k", kind="weights", B=2, Hq=32, Hkv=8, T=500, N=32768, page=64, window=0, sinks=0, cap=0.0, alibi=False, decay=0.0),
        # half of a short cache given up
        dict(name="evict_b1_4k", kind="evict", B=1, Hkv=8, N=4096, keep=2048, sinks=4, recent=256, page=16, W=0),
        # a ragged batch cut to a budget, odd sizes
        dict(name="evict_b8_32k", kind="evict", B=8, Hkv=8, N=32749, keep=8001, sinks=16, recent=1024, page=64, W=0),
        # a contiguous cache with its hash codes, cut to half
        dict(name="evict_b4_128k_codes", kind="evict", B=4, Hkv=8, N=131072, keep=65536, sinks=4, recent=4096, page=0, W=2),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "weights", "weights", "evict", "evict"])
    B, Hkv, G = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([2, 4, 8]), rng.choice([1, 2, 4, 4, 8, 16])
    page = rng.choice([0, 16, 32, 64, 64, 256])
    if kind == "evict":
        N = _log(rng, 64, 4 * 8 * 131072 // (B * Hkv))
        N = min(N, 131072)
        keep = min(N, max(16, _log(rng, max(16, N // 16), N), 1))
        keep = min(keep, 4 * 8 * 65536 // (B * Hkv))
        sinks = rng.randint(0, min(64, keep // 4))
        return dict(kind=kind, B=B, Hkv=Hkv, N=N, keep=keep, sinks=sinks, recent=rng.randint(0, keep // 2), page=page, W=rng.choice([0, 0, 1, 2, 4]))
    G = min(G, 32 // Hkv)
    step = rng.random() < 0.4
    if kind == "weights":
        B = B if step else min(B, 4)
    else:
        B = B if step else min(B, 3)
    T = 1 if step else _log(rng, 2, 8192 if kind == "chunk" else 512)
    most = min(131072, 16 * 8 * 65536 // (B * Hkv), 2 * 32 * 2048 * 32768 // (B * G * Hkv * T))
    if kind == "weights":
        most = min(most, 2 * 32 * 500 * 32768 // (B * G * Hkv * T))
    N = _log(rng, T + 16, max(T + 32, most))
    window = _log(rng, 16, N) if rng.random() < 0.5 else 0
    sinks = rng.randint(0, 128) if window and rng.random() < 0.7 else 0
    cap, alibi = rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), rng.random() < 0.2
    c = dict(kind=kind, B=B, Hq=G * Hkv, Hkv=Hkv, T=T, N=N, page=page, window=window, sinks=sinks, cap=cap, alibi=alibi)
    if kind == "chunk":
        return dict(c, lse=rng.random() < 0.4)
    return dict(c, decay=rng.choice([0.0, 0.9, 1.0, 1.0]))


# ------------------------------------------------- sizes that follow from a case
def _plan(c):
    """(first slot, number of new tokens) of each sequence, ragged."""
    B, T = c["B"], c["T"]
    counts = [T - (2 * T // 3) * b // max(1, B - 1) for b in range(B)]
    most = c["N"] - T
    return [most - (most // 2) * b // max(1, B - 1) for b in range(B)], counts


def _lens(c):
    return [c["N"] - (c["N"] // 2) * b // max(1, c["B"] - 1) for b in range(c["B"])]


def _pairs(c, pos, count):
    """(visible pairs, slots that some token sees) of one sequence."""
    W, S = c["window"], c["sinks"]
    if not W:
        return sum(range(pos + 1, pos + count + 1)), pos + count
    pairs = 0
    for p in range(pos, pos + count):
        lo = max(0, p - W + 1)
        pairs += p + 1 - lo + min(S, lo)
    lo = max(0, pos - W + 1)
    return pairs, pos + count - lo + min(S, lo)


def work(c):
    if c["kind"] == "evict":
        kept = sum(min(n, c["keep"]) for n in _lens(c)) * c["Hkv"]
        return dict(bytes=4 * c["Hkv"] * sum(_lens(c)) + kept * (2 * 2 * D * 2 + 8 * c["W"] + 8), flops=0)
    plan = list(zip(*_plan(c)))
    pairs, seen = (sum(x) for x in zip(*(_pairs(c, *p) for p in plan)))
    rows = c["Hq"] * sum(n for _, n in plan)
    if c["kind"] == "chunk":
        return dict(bytes=rows * (4 * D + 4 * c["lse"]) + seen * c["Hkv"] * 4 * D, flops=c["Hq"] * pairs * 4 * D)
    slots = sum(p + n for p, n in plan)
    return dict(bytes=rows * (2 * D + 4) + seen * c["Hkv"] * 2 * D + slots * c["Hkv"] * (8 if c["decay"] else 4), flops=c["Hq"] * pairs * 2 * D)


# ---------------------------------------------------------------- the inputs
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + tag)
    return g


def _rows(seed, tag, *shape, scale=1.0):
    x = torch.empty(*shape, dtype=torch.bfloat16, device=DEV)
    step = max(1, (1 << 26) // x[0].numel())
    g = _gen(seed, tag)
    for i in range(0, shape[0], step):
        x[i:i + step] = torch.randn(x[i:i + step].shape, generator=g, device=DEV).mul_(scale)
    return x


def _channels(seed, tag, *shape):
    """Rows with a few channels of ten times the scale, as keys have them."""
    x = _rows(seed, tag, *shape)
    x[..., 5::37] *= 10
    return x


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _pages(seed, B, *rows_of, page):
    """Page tables in shuffled order over one pool, one for each of rows_of, and
    the pool's pages: one more than the sequences have."""
    per = [(rows + page - 1) // page for rows in rows_of]
    n = B * sum(per) + 1
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed * 16 + 10)).to(torch.int32)
    tables, at = [], 0
    for p in per:
        tables.append(order[at:at + B * p].view(B, p).to(DEV))
        at += B * p
    return tables, n


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEV)


def _gathered(seed, B, Hkv, N):
    """Weights that slots have gathered: a long tail, and slots that no token
    has looked at, or the same few."""
    x = torch.randn(B, Hkv, N, generator=_gen(seed, 6), device=DEV).mul_(2).exp_()
    return torch.where(x < 0.125, 0.0, torch.where(x < 0.5, 0.25, x))


def prepare(c, seed):
    s = dict(c)
    B, Hkv, N, page = c["B"], c["Hkv"], c["N"], c["page"]
    if c["kind"] == "evict":
        s["lens"] = _ints(_lens(c))
        s["weights"] = _gathered(seed, B, Hkv, N)
        s["weights_out"] = torch.zeros(B, Hkv, c["keep"] + 64, device=DEV)
        if page:  # the kept rows go to other pages of the same pool
            (s["blocks"], s["blocks_out"]), n = _pages(seed, B, N, c["keep"], page=page)
            s["K"], s["V"] = _channels(seed, 1, n, Hkv, page, D), _rows(seed, 2, n, Hkv, page, D)
            s["K_out"], s["V_out"] = s["K"], s["V"]
        else:
            s["blocks"] = s["blocks_out"] = None
            s["K"], s["V"] = _channels(seed, 1, B, Hkv, N, D), _rows(seed, 2, B, Hkv, N, D)
            s["K_out"], s["V_out"] = (torch.zeros(B, Hkv, c["keep"] + 64, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        s["codes"] = s["codes_out"] = None
        if c["W"]:
            s["codes"] = torch.randint(-2 ** 31, 2 ** 31, (B, Hkv, N, c["W"]), generator=_gen(seed, 7), device=DEV, dtype=torch.int32)
            s["codes_out"] = torch.zeros(B, Hkv, c["keep"], c["W"], dtype=torch.int32, device=DEV)
        return s
    T = c["T"]
    pos, counts = _plan(c)
    s["pos"], s["count"] = _ints(pos), _ints(counts)
    s["slopes"] = _slopes(c["Hq"]) if c["alibi"] else None
    # the projection's rows: heads of q of each token
    s["q"] = _rows(seed, 0, B, T, c["Hq"], D, scale=1.5).transpose(1, 2)
    (s["blocks"],), n = _pages(seed, B, N, page=page) if page else ((None,), B)
    s["K"] = _channels(seed, 1, n, Hkv, page or N, D)
    if c["kind"] == "chunk":
        s["V"] = _rows(seed, 2, n, Hkv, page or N, D)
        s["out"] = torch.zeros(B, c["Hq"], T, D, dtype=torch.bfloat16, device=DEV)
        s["lse_out"] = torch.zeros(B, c["Hq"], T, device=DEV) if c["lse"] else None
        return s
    s["weights"] = _gathered(seed, B, Hkv, N)
    z = _scores(s)  # what the attention of the same tokens has left
    top = z.amax(-1, keepdim=True)
    s["lse"] = ((z - top).exp_().sum(-1).log() + top.squeeze(-1))
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _cached(s, x):
    """The rows [B, Hkv, N, D] of each sequence, in the order of its slots."""
    if s["blocks"] is None:
        return x
    return x[s["blocks"].long()].transpose(1, 2).flatten(2, 3)[:, :, :s["N"]]


def _scores(s):
    """Scores [B, Hq, T, N] in 32 bits, -inf where a token does not look."""
    B, Hq, Hkv, T, N = s["B"], s["Hq"], s["Hkv"], s["T"], s["N"]
    K = _cached(s, s["K"]).float()
    # the heads of a group are the rows of one product
    z = torch.matmul(s["q"].float().reshape(B, Hkv, Hq // Hkv * T, D), K.transpose(2, 3).contiguous()).view(B, Hq, T, N)
    z *= 1 / math.sqrt(D)
    if s["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    n, at = torch.arange(N, device=DEV), s["pos"][:, None] + torch.arange(T, device=DEV)
    away = at[..., None] - n  # [B, T, N]
    if s["slopes"] is not None:
        z -= s["slopes"][:, None, None] * away[:, None].float()
    seen = away >= 0
    if s["window"]:
        seen &= (away < s["window"]) | (n < s["sinks"])
    return z.masked_fill_(~seen[:, None], -math.inf)


def _live(s):
    return (torch.arange(s["T"], device=DEV) < s["count"][:, None])[:, None]  # [B, 1, T]


def _plain_chunk(s):
    B, Hq, Hkv, T, N = s["B"], s["Hq"], s["Hkv"], s["T"], s["N"]
    z = _scores(s)
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(B, Hkv, Hq // Hkv * T, N), _cached(s, s["V"]).float()).view(B, Hq, T, D) / total
    live = _live(s)
    out = torch.where(live[..., None], o.to(torch.bfloat16), s["out"])
    if not s["lse"]:
        return out
    return out, torch.where(live, (total.log() + top).squeeze(-1), s["lse_out"])


def _plain_weights(s):
    B, Hq, Hkv, T, N = s["B"], s["Hq"], s["Hkv"], s["T"], s["N"]
    p = _scores(s).sub_(s["lse"][..., None]).exp_()
    p *= _live(s)[..., None]
    gained = p.view(B, Hkv, Hq // Hkv * T, N).sum(2)
    inside = torch.arange(N, device=DEV) < (s["pos"] + s["count"])[:, None]
    old = s["weights"] * s["decay"] if s["decay"] else torch.zeros_like(s["weights"])
    s["weights"].copy_(torch.where(inside[:, None], old + gained, s["weights"]))
    return s["weights"]


def _plain_evict(s):
    B, Hkv, N, keep, page = s["B"], s["Hkv"], s["N"], s["keep"], s["page"]
    n, lens = torch.arange(N, device=DEV), s["lens"][:, None, None]
    key = torch.where((n < s["sinks"]) | (n >= lens - s["recent"]), math.inf, s["weights"])
    key = torch.where(n < lens, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1][..., :keep]
    row = torch.arange(keep, device=DEV)
    valid = (row < lens).expand(B, Hkv, keep)
    kept = torch.sort(torch.where(valid, order, N), dim=-1)[0]
    src = torch.where(valid, kept, 0)
    b, h = torch.arange(B, device=DEV)[:, None, None], torch.arange(Hkv, device=DEV)[:, None]
    if page:
        source, goal = (s["blocks"].long()[b, src // page], h, src % page), (s["blocks_out"].long()[:, None, row // page], h, row % page)
    else:
        source, goal = (b, h, src), (b, h, row)
    for x, y in ((s["K"], s["K_out"]), (s["V"], s["V_out"])):
        y[goal] = torch.where(valid[..., None], x[source], y[goal])
    s["weights_out"].zero_()
    s["weights_out"][..., :keep] = torch.where(valid, s["weights"][b, h, src], 0.0)
    got = [torch.where(valid, kept, -1).to(torch.int32), s["K_out"], s["V_out"], s["weights_out"]]
    if s["codes"] is not None:
        s["codes_out"].copy_(torch.where(valid[..., None], s["codes"][b, h, src], s["codes_out"]))
        got.append(s["codes_out"])
    return got


_plain = dict(chunk=_plain_chunk, weights=_plain_weights, evict=_plain_evict)


def _own_chunk(s):
    import paper_2608_04405_amd as bpc
    out = bpc.chunk_attention(s["q"], s["K"], s["V"], s["pos"], count=s["count"], N=s["N"], block_table=s["blocks"], window=s["window"],
                              sinks=s["sinks"], softcap=s["cap"], slopes=s["slopes"], out=s["out"], lse_out=s["lse_out"])
    return (out, s["lse_out"]) if s["lse"] else out


def _own_weights(s):
    import paper_2608_04405_amd as bpc
    return bpc.key_weights(s["q"], s["K"], s["lse"], s["weights"], s["pos"], count=s["count"], N=s["N"], block_table=s["blocks"],
                           window=s["window"], sinks=s["sinks"], softcap=s["cap"], slopes=s["slopes"], decay=s["decay"])


def _own_evict(s):
    import paper_2608_04405_amd as bpc
    kept = bpc.evict_kv(s["K"], s["V"], s["weights"], s["lens"], s["keep"], s["K_out"], s["V_out"], sinks=s["sinks"], recent=s["recent"],
                        block_table=s["blocks"], table_out=s["blocks_out"], codes=s["codes"], codes_out=s["codes_out"],
                        weights_out=s["weights_out"])
    got = [kept, s["K_out"], s["V_out"], s["weights_out"]]
    return got if s["codes"] is None else got + [s["codes_out"]]


_own = dict(chunk=_own_chunk, weights=_own_weights, evict=_own_evict)


# ---------------------------------------------------------------- in 64 bits
def _exact_rows(c, s, b, h, x):
    """Slots of one head of one sequence in 64 bits, found one index at a time."""
    n = torch.arange(c["N"], device=DEV)
    if not c["page"]:
        return x[b, h].double()
    return x[s["blocks"][b].long()[n // c["page"]], h, n % c["page"]].double()


def _exact_scores(c, s, b, j, k, pos, count):
    """Scores [count, N] of query head j of sequence b."""
    z = s["q"][b, j, :count].double() @ k.t() / D ** 0.5
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    n, p = torch.arange(c["N"], device=DEV), torch.arange(pos, pos + count, device=DEV)[:, None]
    if c["alibi"]:
        z = z + (n - p) * float(s["slopes"][j])
    hidden = n > p
    if c["window"]:
        hidden |= (n <= p - c["window"]) & (n >= c["sinks"])
    z[hidden] = -math.inf
    return z


def _exact_evict(c, s):
    B, Hkv, keep, page = c["B"], c["Hkv"], c["keep"], c["page"]
    kept = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device=DEV)
    K, V = s["K_out"].double(), s["V_out"].double()
    weights = torch.zeros(s["weights_out"].shape, dtype=torch.float64, device=DEV)
    codes = None if s["codes_out"] is None else s["codes_out"].clone()
    for b, n in enumerate(_lens(c)):
        m = min(n, keep)
        for h in range(Hkv):
            w = s["weights"][b, h, :n].double()
            if n <= keep:
                best = torch.arange(n, device=DEV)
            else:
                first, last = c["sinks"], n - c["recent"]
                free = keep - first - c["recent"]
                mid = w[first:last]
                # the value of the last one taken, all above it, and the first ones that equal it
                least = torch.topk(mid, free)[0][-1] if free else math.inf
                above, same = mid > least, (mid == least).nonzero()[:, 0]
                taken = above.clone()
                taken[same[:free - int(above.sum())]] = True
                best = torch.cat([torch.arange(first, device=DEV), taken.nonzero()[:, 0] + first, torch.arange(last, n, device=DEV)])
            kept[b, h, :m] = best.to(torch.int32)
            weights[b, h, :m] = w[best]
            row = torch.arange(m, device=DEV)
            for x, y in ((s["K"], K), (s["V"], V)):
                if page:
                    y[s["blocks_out"][b].long()[row // page], h, row % page] = x[s["blocks"][b].long()[best // page], h, best % page].double()
                else:
                    y[b, h, :m] = x[b, h][best].double()
            if codes is not None:
                codes[b, h, :m] = s["codes"][b, h][best]
    got = [kept, K, V, weights]
    return got if codes is None else got + [codes]


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "evict":
        return _exact_evict(c, s)
    G = c["Hq"] // c["Hkv"]
    pos, counts = _plan(c)
    if c["kind"] == "weights":
        total = s["weights"].double()
        for b in range(c["B"]):
            end = pos[b] + counts[b]
            total[b, :, :end] *= c["decay"]
            for j in range(c["Hq"]):
                if j % G == 0:
                    k = _exact_rows(c, s, b, j // G, s["K"])
                z = _exact_scores(c, s, b, j, k, pos[b], counts[b])
                total[b, j // G, :end] += torch.exp(z - s["lse"][b, j, :counts[b], None].double()).sum(0)[:end]
        return total
    out = torch.zeros(c["B"], c["Hq"], c["T"], D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["B"], c["Hq"], c["T"], dtype=torch.float64, device=DEV)
    for b in range(c["B"]):
        for j in range(c["Hq"]):
            if j % G == 0:
                k, v = (_exact_rows(c, s, b, j // G, s[x]) for x in ("K", "V"))
            z = _exact_scores(c, s, b, j, k, pos[b], counts[b])
            lse[b, j, :counts[b]] = torch.logsumexp(z, -1)
            out[b, j, :counts[b]] = torch.softmax(z, -1) @ v
    return (out, lse) if c["lse"] else out
