"""Timed cases of the operators around the hashed cache: what makes its queries
and keys (``qk_norm_rope``), writes them to a paged cache (``append_kv_paged``),
attends at prefill (``prefill_attention``) and verifies drafted tokens over the
cache (``tree_attention``), with their plain forms in torch.

Head dim is 128 throughout, tensors are bf16.  With ``own`` set, ``run`` makes
the framework's calls; otherwise it computes the same in elementary torch
operations in 32 bits, rounded once at the end.  ``exact`` is the definition in
64 bits.
"""

import math

import torch

own = False

D = 128
DEV = "cuda"
EPS = 1e-6


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one token of one request: launch latency
        dict(name="qk_step_b1", kind="qk", B=1, T=1, Hq=32, Hkv=8, R=128, interleaved=False, norm=True, fused=True),
        # the prefill of one long request of odd length, views of the fused projection
        dict(name="qk_prefill_32749", kind="qk", B=1, T=32749, Hq=32, Hkv=8, R=128, interleaved=False, norm=True, fused=True),
        # the token that each sequence of a batch appends before its step
        dict(name="append_step_b16", kind="append", B=16, T=1, Hkv=8, page=16, top=4096, R=128, interleaved=False, norm=False, tree=False),
        # a tree of drafted tokens for each sequence, half of each head rotated by depth in adjacent pairs
        dict(name="append_tree_b16_24", kind="append", B=16, T=24, Hkv=8, page=64, top=8192, R=64, interleaved=True, norm=True, tree=True),
        # a prefill chunk of a batch with ragged lengths
        dict(name="append_chunk_b4_8192", kind="append", B=4, T=8192, Hkv=8, page=256, top=16384, R=128, interleaved=False, norm=True, tree=False),
        # a short prompt
        dict(name="prefill_257", kind="prefill", B=1, Hq=8, Hkv=2, T=257, N=257, cap=0.0, alibi=False, mask="causal"),
        # a batch of causal prefills
        dict(name="prefill_b2_8k", kind="prefill", B=2, Hq=32, Hkv=8, T=8192, N=8192, cap=0.0, alibi=False, mask="causal"),
        # packed documents with padding behind the last, capped scores
        dict(name="prefill_docs_8001_cap", kind="prefill", B=1, Hq=32, Hkv=8, T=8001, N=8001, cap=50.0, alibi=False, mask="documents"),
        # a chunk over a long cache behind a prefix that sees itself, distance bias
        dict(name="prefill_chunk_512_64k_bias", kind="prefill", B=1, Hq=32, Hkv=8, T=512, N=65536, cap=0.0, alibi=True, mask="prefix"),
        # one token over a short paged cache: launch latency
        dict(name="tree_step_b1_4k", kind="tree", B=1, Hq=32, Hkv=8, T=1, N=4096, page=16, cap=0.0, alibi=False, tree=False),
        # drafted trees of a ragged batch over a paged cache, capped scores and a distance bias
        dict(name="tree_b8_24_32k_cap_bias", kind="tree", B=8, Hq=32, Hkv=8, T=24, N=32768, page=64, cap=30.0, alibi=True, tree=True),
        # a batch at long context in the contiguous cache, a chain of eight drafts
        dict(name="tree_b16_8_128k", kind="tree", B=16, Hq=32, Hkv=8, T=8, N=131072, page=0, cap=0.0, alibi=False, tree=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["qk", "append", "prefill", "prefill", "tree", "tree"])
    B, Hkv, G = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([2, 4, 8]), rng.choice([1, 2, 4, 4, 8, 16])
    if kind in ("qk", "append"):
        R, inter = rng.choice([32, 64, 128, 128]), rng.random() < 0.3
        if kind == "qk":
            G = min(G, 32 // Hkv)
            return dict(kind=kind, B=B, T=_log(rng, 1, 32768 // B), Hq=G * Hkv, Hkv=Hkv, R=R, interleaved=inter, norm=rng.random() < 0.6,
                        fused=rng.random() < 0.5)
        tree = rng.random() < 0.4
        T = rng.randint(2, 64) if tree else _log(rng, 1, 32768 // B)
        return dict(kind=kind, B=B, T=T, Hkv=Hkv, page=rng.choice([16, 32, 64, 128, 256]), top=T + _log(rng, 16, 8192), R=R,
                    interleaved=inter, norm=rng.random() < 0.5, tree=tree)
    cap, alibi = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3
    if kind == "prefill":
        B, G = min(B, 3), min(G, 32 // Hkv)
        T = _log(rng, 1, 8192)
        N = T if rng.random() < 0.6 else min(65536, T + _log(rng, 1, 32768))
        N = max(T, min(N, 2 * 8192 * 8192 * 32 // (B * G * Hkv * T)))
        return dict(kind=kind, B=B, Hq=G * Hkv, Hkv=Hkv, T=T, N=N, cap=cap, alibi=alibi, mask=rng.choice(["causal", "documents", "prefix"]))
    T = rng.choice([1, 1, rng.randint(2, 64), rng.randint(2, 64)])
    N = _log(rng, T + 64, max(T + 128, min(131072, 16 * 8 * 131072 // (B * Hkv), 16 * 32 * 8 * 131072 // (B * G * Hkv * T))))
    return dict(kind=kind, B=B, Hq=G * Hkv, Hkv=Hkv, T=T, N=N, page=rng.choice([0, 16, 32, 64, 256]), cap=cap, alibi=alibi, tree=T > 1 and rng.random() < 0.7)


# ------------------------------------------------- sizes that follow from a case
def _tree_lens(c):
    """Cached tokens of each sequence: from half the longest to the longest."""
    most = c["N"] - c["T"]
    return [most - (most // 2) * b // max(1, c["B"] - 1) for b in range(c["B"])]


def _append_plan(c):
    """(first slot, number of new tokens) of each sequence."""
    counts = [c["T"] - (c["T"] // 3) * b // max(1, c["B"] - 1) for b in range(c["B"])]
    return [(c["top"] - c["T"]) * (b + 1) // c["B"] for b in range(c["B"])], counts


def _doc_lengths(c):
    """Lengths of packed documents, ragged, and of the padding behind the last."""
    pad = min(c["N"] // 32, c["T"] // 2)
    left, out, i = c["N"] - pad, [], 0
    while left:
        n = min(left, max(1, c["N"] * (1 + (i * 5) % 7) // 24 + i % 3))
        out.append(n)
        left, i = left - n, i + 1
    return out, pad


def _ranges(c):
    """Visible keys [begin, end) of each query of a prefill, as lists."""
    T, N, pos0 = c["T"], c["N"], c["N"] - c["T"]
    if c["mask"] == "causal":
        return [0] * T, [pos0 + t + 1 for t in range(T)]
    if c["mask"] == "prefix":
        prefix = N - T // 2
        return [0] * T, [max(pos0 + t + 1, prefix) for t in range(T)]
    docs, pad = _doc_lengths(c)
    first, end, n0 = [], [], 0
    for n in docs:
        first += [n0] * n
        end += range(n0 + 1, n0 + n + 1)
        n0 += n
    return (first + [0] * pad)[pos0:], (end + [0] * pad)[pos0:]


def work(c):
    if c["kind"] == "qk":
        rows = c["B"] * c["T"] * (c["Hq"] + c["Hkv"])
        # each row in and out, the tokens' table rows and positions
        table = c["T"] * c["R"] * 4
        return dict(bytes=rows * 2 * D * 2 + table + c["B"] * c["T"] * 4, flops=rows * (3 * c["R"] + (4 * D if c["norm"] else 0)))
    if c["kind"] == "append":
        _, counts = _append_plan(c)
        tokens = sum(counts)
        return dict(bytes=tokens * (c["Hkv"] * 4 * D * 2 + c["R"] * 4), flops=tokens * c["Hkv"] * (3 * c["R"] + (4 * D if c["norm"] else 0)))
    if c["kind"] == "prefill":
        first, end = _ranges(c)
        pairs = sum(e - f for f, e in zip(first, end) if e > f)
        return dict(bytes=c["B"] * 2 * D * (2 * c["Hq"] * c["T"] + 2 * c["Hkv"] * c["N"]), flops=c["B"] * c["Hq"] * pairs * 4 * D)
    lens = _tree_lens(c)
    keys = sum(lens) + c["B"] * c["T"]
    return dict(bytes=2 * D * (2 * c["Hkv"] * keys + 2 * c["B"] * c["Hq"] * c["T"]), flops=4 * D * c["Hq"] * c["T"] * sum(lens))


# ---------------------------------------------------------------- the inputs
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + tag)
    return g


def _rows(seed, tag, *shape, scale=1.0):
    x = torch.empty(*shape, dtype=torch.bfloat16, device=DEV)
    g = _gen(seed, tag)
    for i in range(shape[0]):
        x[i] = torch.randn(*shape[1:], generator=g, device=DEV).mul_(scale)
    return x


def _channels(seed, tag, *shape):
    """Rows with a few channels of ten times the scale, as keys have them."""
    x = _rows(seed, tag, *shape)
    x[..., 5::37] *= 10
    return x


def _table(rows, R):
    """cos and sin of every position, [rows, R] fp32, cosines first."""
    angle = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R)
    return torch.cat([angle.cos(), angle.sin()], -1).float()


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _parents(seed, B, T):
    """A random tree of T drafts for each sequence: ancestor bits and depths."""
    g = torch.Generator().manual_seed(seed * 16 + 9)
    pick = torch.rand(B, T, generator=g).tolist()
    bits, depth = [[0] * T for _ in range(B)], [[0] * T for _ in range(B)]
    for b in range(B):
        for t in range(1, T):
            p = int(pick[b][t] * t) // 2  # early drafts have the more children
            bits[b][t], depth[b][t] = bits[b][p] | 1 << p, depth[b][p] + 1
    signed = [[(x | 1 << t) - (1 << 64 if t == 63 else 0) for t, x in enumerate(r)] for r in bits]
    return torch.tensor(signed, dtype=torch.int64, device=DEV), torch.tensor(depth, dtype=torch.int32, device=DEV)


def _pages(seed, B, rows, page):
    """A page table in shuffled order, one spare page that no sequence has."""
    per = (rows + page - 1) // page
    order = torch.randperm(B * per + 1, generator=torch.Generator().manual_seed(seed * 16 + 10))
    return order[:B * per].view(B, per).to(torch.int32).to(DEV), B * per + 1


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEV)


def prepare(c, seed):
    s = dict(c)
    B, T, Hkv = c["B"], c["T"], c["Hkv"]
    if c["kind"] == "qk":
        H = c["Hq"] + 2 * Hkv
        if c["fused"]:  # the fused projection's rows: heads of q, then k, then v
            x = _channels(seed, 0, B, T, H, D)
            s["q"], s["k"] = x[:, :, :c["Hq"]].transpose(1, 2), x[:, :, c["Hq"]:c["Hq"] + Hkv].transpose(1, 2)
        else:
            s["q"], s["k"] = _channels(seed, 0, B, c["Hq"], T, D), _channels(seed, 1, B, Hkv, T, D)
        s["table"] = _table(T + 64, c["R"])
        s["pos"] = torch.arange(T, device=DEV, dtype=torch.int32)[None] + _ints([[7 * b % 61] for b in range(B)])
    elif c["kind"] == "append":
        s["k"], s["v"] = _channels(seed, 0, B, T, Hkv, D).transpose(1, 2), _rows(seed, 1, B, T, Hkv, D).transpose(1, 2)
        s["blocks"], n = _pages(seed, B, c["top"], c["page"])
        s["K"], s["V"] = _rows(seed, 2, n, Hkv, c["page"], D), _rows(seed, 3, n, Hkv, c["page"], D)
        pos, counts = _append_plan(c)
        s["pos"], s["count"] = _ints(pos), _ints(counts)
        s["table"] = _table(c["top"], c["R"])
        s["rope_pos"] = s["pos"][:, None] + _parents(seed, B, T)[1] if c["tree"] else None
    else:
        s["q"] = _rows(seed, 0, B, c["Hq"], T, D, scale=1.5)
        s["slopes"] = _slopes(c["Hq"]) if c["alibi"] else None
        if c["kind"] == "prefill":
            s["K"], s["V"] = _channels(seed, 1, B, Hkv, c["N"], D), _rows(seed, 2, B, Hkv, c["N"], D)
            begin, end = _ranges(c)
            plain = c["mask"] == "causal"
            s["begin"] = None if plain else _ints(begin).expand(B, T).contiguous()
            s["end"] = None if plain else _ints(end).expand(B, T).contiguous()
        else:
            s["lens"] = _ints(_tree_lens(c))
            s["tree"] = _parents(seed, B, T)[0] if c["tree"] else None
            s["blocks"], n = _pages(seed, B, c["N"], c["page"]) if c["page"] else (None, B)
            s["K"], s["V"] = _channels(seed, 1, n, Hkv, c["page"] or c["N"], D), _rows(seed, 2, n, Hkv, c["page"] or c["N"], D)
    if c.get("norm"):
        s["wq"], s["wk"] = ((1 + 0.1 * torch.randn(D, generator=_gen(seed, t), device=DEV)).to(torch.bfloat16) for t in (4, 5))
    else:
        s["wq"] = s["wk"] = None
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _plain_rows(x, w, table, pos, R, interleaved):
    """Norm and rotation of x [B, H, T, D] at pos [B, T], in 32 bits."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    cs = table[pos.long()][:, None]
    c, sn = cs[..., :R // 2], cs[..., R // 2:]
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([turned, x[..., R:]], -1).to(torch.bfloat16)


def _plain_qk(s):
    return tuple(_plain_rows(s[x], s["w" + x], s["table"], s["pos"], s["R"], s["interleaved"]) for x in ("q", "k"))


def _plain_append(s):
    T, page = s["T"], s["page"]
    step = torch.arange(T, device=DEV)
    slot = (s["pos"].long()[:, None] + step).clamp(max=s["blocks"].shape[1] * page - 1)
    new = (step < s["count"][:, None])[..., None, None]
    at = torch.gather(s["blocks"].long(), 1, slot // page), slot % page  # [B, T]
    turn = slot if s["rope_pos"] is None else s["rope_pos"]
    k = _plain_rows(s["k"], s["wk"], s["table"], turn.clamp(max=s["table"].shape[0] - 1), s["R"], s["interleaved"])
    s["K"][at[0], :, at[1]] = torch.where(new, k.transpose(1, 2), s["K"][at[0], :, at[1]])
    s["V"][at[0], :, at[1]] = torch.where(new, s["v"].transpose(1, 2), s["V"][at[0], :, at[1]])
    return s["K"], s["V"]


def _plain_attend(q, K, V, cap, slopes, distance, seen):
    """q [B, Hq, T, D] over K, V [B, Hkv, N, D]; distance and seen [B, T, N]."""
    B, Hq, T, _ = q.shape
    Hkv, N = K.shape[1], K.shape[2]
    # the heads of a group are the rows of one product
    z = torch.matmul(q.float().reshape(B, Hkv, Hq // Hkv * T, D), K.float().transpose(2, 3).contiguous()).view(B, Hq, T, N)
    z *= 1 / math.sqrt(D)
    if cap:
        z = cap * torch.tanh(z / cap)
    if slopes is not None:
        z -= slopes[:, None, None] * distance[:, None].float()
    z = torch.where(seen[:, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    z = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(B, Hkv, Hq // Hkv * T, N), V.float()).view(B, Hq, T, D)
    return torch.where(total == 0, 0.0, o / total).to(torch.bfloat16)


def _plain_prefill(s):
    T, N = s["T"], s["N"]
    key, at = torch.arange(N, device=DEV), torch.arange(N - T, N, device=DEV)
    if s["end"] is None:
        seen = (key <= at[:, None])[None]
    else:
        seen = (key >= s["begin"][..., None]) & (key < s["end"][..., None])
    distance = (at[:, None] - key).abs()[None]
    return _plain_attend(s["q"], s["K"], s["V"], s["cap"], s["slopes"], distance, seen)


def _plain_tree(s):
    B, T, N = s["B"], s["T"], s["N"]
    K, V = s["K"], s["V"]
    if s["blocks"] is not None:
        K, V = (x[s["blocks"].long()].transpose(1, 2).flatten(2, 3)[:, :, :N] for x in (K, V))
    key, draft, lens = torch.arange(N, device=DEV), torch.arange(T, device=DEV), s["lens"].long()[:, None]
    if s["tree"] is None:
        sees = (draft <= draft[:, None]).expand(B, T, T)
    else:
        sees = (s["tree"][..., None] >> draft & 1).bool()
    depth = (sees & (draft != draft[:, None])).sum(-1)
    j = key - lens  # the draft that a key belongs to
    seen = (j < 0)[:, None] | ((j >= 0) & (j < T))[:, None] & torch.gather(sees, 2, j.clamp(0, T - 1)[:, None].expand(B, T, N))
    place = torch.where(j < 0, key, lens + torch.gather(depth, 1, j.clamp(0, T - 1)))
    distance = (lens + depth)[..., None] - place[:, None]
    return _plain_attend(s["q"], K, V, s["cap"], s["slopes"], distance.abs(), seen)


_plain = dict(qk=_plain_qk, append=_plain_append, prefill=_plain_prefill, tree=_plain_tree)


def _own_qk(s):
    import paper_2608_04405_amd as bpc
    return bpc.qk_norm_rope(s["q"], s["k"], s["pos"], s["table"], wq=s["wq"], wk=s["wk"], eps=EPS, interleaved=s["interleaved"])


def _own_append(s):
    import paper_2608_04405_amd as bpc
    bpc.append_kv_paged(s["k"], s["v"], s["K"], s["V"], s["blocks"], s["pos"], count=s["count"], cos_sin=s["table"], rope_pos=s["rope_pos"],
                        wk=s["wk"], eps=EPS, interleaved=s["interleaved"])
    return s["K"], s["V"]


def _own_prefill(s):
    import paper_2608_04405_amd as bpc
    return bpc.prefill_attention(s["q"], s["K"], s["V"], softcap=s["cap"], slopes=s["slopes"], key_begin=s["begin"], key_end=s["end"])


def _own_tree(s):
    import paper_2608_04405_amd as bpc
    return bpc.tree_attention(s["q"], s["K"], s["V"], s["lens"], s["tree"], N=s["N"], block_table=s["blocks"], softcap=s["cap"], slopes=s["slopes"])


_own = dict(qk=_own_qk, append=_own_append, prefill=_own_prefill, tree=_own_tree)


# ---------------------------------------------------------------- in 64 bits
def _exact_turn(x, w, table, pos, R, interleaved):
    """Row vectors as complex numbers: pair times (cos + i sin)."""
    x = x.double()
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
    head, rest = x[..., :R], x[..., R:]
    if interleaved:
        pair = head.unflatten(-1, (R // 2, 2)).contiguous()
    else:
        pair = head.unflatten(-1, (2, R // 2)).transpose(-1, -2).contiguous()
    cs = table.double().unflatten(-1, (2, R // 2)).transpose(-1, -2).contiguous()
    turned = torch.view_as_real(torch.view_as_complex(pair) * torch.view_as_complex(cs)[pos.long()].unsqueeze(1))
    turned = turned.flatten(-2) if interleaved else turned.transpose(-1, -2).flatten(-2)
    return torch.cat([turned, rest], -1)


def _exact_attention(q, K, V, cap, slopes, mask, distance):
    """A query head at a time."""
    B, Hq, T, _ = q.shape
    G = Hq // K.shape[1]
    out = torch.zeros(B, Hq, T, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        gone = ~mask[b % mask.shape[0]]
        empty = gone.all(-1, keepdim=True)
        for h in range(K.shape[1]):
            k, v = K[b, h].double().t().contiguous(), V[b, h].double()
            for g in range(h * G, h * G + G):
                score = q[b, g].double() @ k / D ** 0.5
                if cap:
                    score = torch.tanh(score / cap) * cap
                if slopes is not None:
                    score = score - slopes[g].double() * distance[b % distance.shape[0]]
                out[b, g] = torch.softmax(score.masked_fill(gone, -math.inf), -1).masked_fill(empty, 0) @ v
    return out


def exact(c, seed):
    s = prepare(c, seed)
    B, T = c["B"], c["T"]
    if c["kind"] == "qk":
        return tuple(_exact_turn(s[x], s["w" + x], s["table"], s["pos"], c["R"], c["interleaved"]) for x in ("q", "k"))
    if c["kind"] == "append":
        K, V = s["K"].double(), s["V"].double()
        pos, counts = _append_plan(c)
        for b in range(B):
            n = counts[b]
            slots = torch.arange(pos[b], pos[b] + n, device=DEV)
            turn = slots if s["rope_pos"] is None else s["rope_pos"][b, :n]
            k = _exact_turn(s["k"][b:b + 1, :, :n], s["wk"], s["table"], turn[None], c["R"], c["interleaved"])[0]
            page = s["blocks"][b].long()[slots // c["page"]]
            K[page, :, slots % c["page"]] = k.transpose(0, 1)
            V[page, :, slots % c["page"]] = s["v"][b, :, :n].double().transpose(0, 1)
        return K, V
    N = c["N"]
    n = torch.arange(N, device=DEV)
    if c["kind"] == "prefill":
        begin, end = (_ints(x) for x in _ranges(c))
        mask = ((begin[:, None] <= n) & (n < end[:, None]))[None]
        distance = (n - torch.arange(N - T, N, device=DEV)[:, None]).abs()[None]
        return _exact_attention(s["q"], s["K"], s["V"], c["cap"], s["slopes"], mask, distance)
    mask, distance = torch.zeros(B, T, N, dtype=torch.bool, device=DEV), torch.zeros(B, T, N, dtype=torch.int32, device=DEV)
    K, V = s["K"], s["V"]
    if c["page"]:
        rows = (s["blocks"].long()[:, n // c["page"]], n % c["page"])  # [B, N], [N]
        K, V = (x[rows[0], :, rows[1]].transpose(1, 2) for x in (K, V))
    for b, L in enumerate(_tree_lens(c)):
        mask[b, :, :L] = True
        sees = torch.tensor([[x >> j & 1 for j in range(T)] for x in s["tree"][b].tolist()]) if c["tree"] else torch.ones(T, T).tril()
        mask[b, :, L:L + T] = sees.bool().to(DEV)
        level = (sees.sum(-1) - 1).to(torch.int32).to(DEV)
        where = torch.cat([n[:L], L + level, n[L + T:]])
        distance[b] = (L + level)[:, None] - where
    return _exact_attention(s["q"], K, V, c["cap"], s["slopes"], mask, distance.abs_())
