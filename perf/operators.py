"""The operators of the block-scaled FP8 KV cache, as programs call them: the
calls, their plain forms, and their results in 64 bits.

A cache holds one layer's K and V of one sequence in OCP E4M3, one power-of-two
scale for every block of 64 rows and KV head, and for K the lowest and highest
code of every channel of a block ("bounds").  The rows of the last block, while
it is not full, are also kept in bf16 ("open"), since its scale may still grow.

  append   T new rows of K and V enter the cache
  attend   causal attention of the T newest tokens over the cache
  sparse   the same over the n_sel blocks that the bounds select for each token
           and KV head: selection, then attention

A step covers a batch of sequences of their own lengths n, each with T tokens
at positions [n - T, n); q, K, V and o are packed [sum of T, heads, d].

``listed`` gives the fixed cases, ``draw`` more of the same ranges, ``prepare``
what the program holds before the call, ``run`` one pass, ``work`` the bytes and
operations that it cannot do without, ``exact`` its results in 64 bits.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 64
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # one decode token of each of the 32 robot environments (one KV head of
        # 256, 816 rows) enters their caches
        _case("append_step_32_envs", "append", n="816*32", T="1*32", Hkv=1, d=256),
        # one layer's K/V of the 48-layer stack, the whole 16k prefix
        _case("append_16k", "append", n="16384", T="16384", Hkv=4, d=256),
        # suffixes of four sessions of the 8-layer stack, begun and ended inside
        # blocks
        _case("append_ragged", "append", n="2111,8191,4159,67", T="161,2047,33,67", Hkv=4, d=128),
        # decode, the smallest model: 200 rows, 4 KV heads of 64
        _case("decode_200_d64", "attend", n="200", T="1", Hkv=4, G=2, d=64),
        # decode of the 32 robot environments
        _case("decode_32_envs", "attend", n="816*32", T="1*32", Hkv=1, G=8, d=256),
        # decode of one session of the 48-layer stack behind its 16k prefix
        _case("decode_16k", "attend", n="16385", T="1", Hkv=4, G=8, d=256),
        # decode of four sessions, from a fresh one to a long one
        _case("decode_ragged_131k", "attend", n="131072,16449,2111,1", T="1*4", Hkv=4, G=8, d=256),
        # prefill of the 8-layer stack's 2k prefix
        _case("prefill_2k", "attend", n="2048", T="2048", Hkv=4, G=4, d=128),
        # the remainder after a restore at 16384: few queries, many keys
        _case("resume_161_at_16k", "attend", n="16545", T="161", Hkv=4, G=8, d=256),
        # cold prefill of the 48-layer stack's prefix
        _case("prefill_16k", "attend", n="16384", T="16384", Hkv=4, G=8, d=256),
        # sparse decode behind the 16k prefix: 32 of 257 blocks
        _case("sparse_16k", "sparse", n="16385", T="1", Hkv=4, G=8, d=256, n_sel=32),
        # sparse decode of four sessions with a few draft tokens each, one long
        _case("sparse_ragged_131k", "sparse", n="131072,16449,8448,700", T="1,4,3,5", Hkv=4, G=8, d=256, n_sel=64),
    ]


def _case(name, kind, n, T, Hkv, d, G=1, n_sel=0, first=1, last=2):
    """n and T: a number for each sequence, as text ("816*32": 32 times 816)."""
    return {"name": name, "kind": kind, "n": n, "T": T, "Hkv": Hkv, "G": G, "d": d, "n_sel": n_sel, "first": first,
            "last": last}


def _ints(text):
    return [int(a.split("*")[0]) for a in text.split(",") for _ in range(int(a.split("*")[1]) if "*" in a else 1)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: batches of 1 to 32 sequences of 1 to 131072 rows, 1 to 8 KV
    heads of 64, 128 or 256, 1 to 16 query heads to each, one token or many."""
    kind = rng.choice(["append", "attend", "attend", "attend", "sparse"])
    d, Hkv, G = rng.choice([64, 128, 256]), rng.choice([1, 2, 3, 4, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    if kind == "append":
        B = _log_int(rng, 1, 32)
        T = [_log_int(rng, 1, 16384 // B) if rng.random() < 0.6 else 1 for _ in range(B)]
        n = [t + _log_int(rng, 1, 4096) - 1 for t in T]
        G = 1
    elif kind == "attend" and rng.random() < 0.5:  # prefill or a remainder
        B = rng.choice([1, 1, 1, 2, 3])
        T = [_log_int(rng, 2, 8192) for _ in range(B)]
        n = [min(131072, t + _log_int(rng, 1, 16384) - 1) for t in T]
        most = 4.0e12 / (4 * Hkv * G * d)  # no more than the largest listed call
        while sum(t * m for t, m in zip(T, n)) > most:
            n = [max(t, m // 2) for t, m in zip(T, n)]
            T = [max(1, min(t, m, t * 3 // 4)) for t, m in zip(T, n)]
    else:  # decode, one token or a few draft tokens
        B = _log_int(rng, 1, 32)
        T = [1] * B if rng.random() < 0.6 else [rng.randint(1, 6) for _ in range(B)]
        n = [max(t, _log_int(rng, 1, 131072)) for t in T]
        rows = 150000 * 1024 // (Hkv * d)
        while sum(n) > rows:
            n = [max(t, m // 2) for t, m in zip(T, n)]
    c = _case("", kind, ",".join(map(str, n)), ",".join(map(str, T)), Hkv, d, G, _log_int(rng, 4, 96) if kind == "sparse" else 0,
              rng.choice([0, 1, 1]), rng.choice([1, 2, 3]))
    del c["name"]
    return c


# ---------------------------------------------------------------- prepare --
def _encode(x, e):
    """E4M3 codes of x / 2^e: nearest, ties to even, saturated; NaN stays."""
    return torch.ldexp(x.float(), -e).clamp(-448.0, 448.0).to(E4M3)


def _exponent(amax):
    """The smallest e with amax <= 448 * 2^e, within [-100, 119]."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x - torch.where(m <= 0.875, 9, 8), -100).clamp(-100, 119)


def _blocks(x):
    """Codes [B, rows, Hkv, d], scales [B, nb, Hkv] and bounds [B, nb, 2, Hkv, d] of the rows x from the start of a block on."""
    rows = x.shape[1]
    nb = -(-rows // BLOCK)
    y = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, nb * BLOCK - rows)).unflatten(1, (nb, BLOCK))
    held = (torch.arange(nb * BLOCK, device=x.device) < rows).view(nb, BLOCK, 1, 1)
    e = _exponent(torch.where(y.isfinite(), y.abs(), 0.0).amax((2, 4)))
    at = e[:, :, None, :, None]
    lo = torch.where(held, y, math.inf).amin(2, keepdim=True)
    hi = torch.where(held, y, -math.inf).amax(2, keepdim=True)
    bounds = torch.cat([_encode(lo, at), _encode(hi, at)], 2)
    return _encode(y, at).flatten(1, 2)[:, :rows], torch.ldexp(torch.ones_like(e, dtype=torch.float32), e), bounds


def _put(s, g, x, side, b0):
    """Rows x [B, rows, Hkv, d] of K (side 0) or V (side 1) of the sequences of group g, from the start of block b0 on,
    enter their caches."""
    codes, scales, bounds = _blocks(x)
    r0 = s["row0"][g["at"], None] + b0 * BLOCK
    s["kv"][side][r0 + torch.arange(x.shape[1], device="cuda")] = codes.view(torch.uint8)
    blocks = r0 // BLOCK + torch.arange(scales.shape[1], device="cuda")
    s["scales"][blocks, side] = scales
    if side == 0:
        s["bounds"][blocks] = bounds.view(torch.uint8)
    tail = x.shape[1] % BLOCK
    if tail:
        s["open"][g["at"], side, :tail] = x[:, -tail:]


def prepare(case, seed):
    c = case
    n, T, Hkv, G, d = _ints(c["n"]), _ints(c["T"]), c["Hkv"], c["G"], c["d"]
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    cap = [(-(-m // BLOCK) + 1) * BLOCK for m in n]  # rows of each cache
    row0, token0 = ([sum(x[:i]) for i in range(len(n))] for x in (cap, T))
    rows, tokens = sum(cap), sum(T)
    # keys have a few channels of large values and an offset, as models' keys do; values are of mixed size by head
    chan = torch.exp(0.5 * normal(1, Hkv, d))
    mean = 0.5 * normal(1, Hkv, d) * chan
    s = {"case": c, "scale": 1.0 / math.sqrt(d), "row0": torch.tensor(row0, device="cuda"),
         # sequences of the same lengths, which the plain form takes together
         "groups": [{"n": m, "T": t, "at": [i for i in range(len(n)) if (n[i], T[i]) == (m, t)]} for m, t in dict.fromkeys(zip(n, T))],
         "kv": [torch.zeros((rows, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2)],
         "scales": torch.zeros((rows // BLOCK, 2, Hkv), dtype=torch.float32, device="cuda"),
         "bounds": torch.zeros((rows // BLOCK, 2, Hkv, d), dtype=torch.uint8, device="cuda"),
         "open": torch.zeros((len(n), 2, BLOCK, Hkv, d), dtype=torch.bfloat16, device="cuda")}
    for g in s["groups"]:
        B, m = len(g["at"]), g["n"] - (g["T"] if c["kind"] == "append" else 0)
        g["tokens"] = torch.tensor([token0[i] for i in g["at"]], device="cuda")[:, None] + torch.arange(g["T"], device="cuda")
        if m:
            _put(s, g, (mean + chan * normal(B, m, Hkv, d)).bfloat16(), 0, 0)
            _put(s, g, (torch.exp(normal(1, 1, Hkv, 1)) * normal(B, m, Hkv, d)).bfloat16(), 1, 0)
    # one record for each sequence: addresses of its buffers, its capacity, rows held with the step's tokens, tokens
    s["seqs"] = np.array([[s["kv"][0].data_ptr() + r * Hkv * d, s["kv"][1].data_ptr() + r * Hkv * d,
                           s["scales"].data_ptr() + r // BLOCK * 2 * Hkv * 4, s["bounds"].data_ptr() + r // BLOCK * 2 * Hkv * d,
                           s["open"].data_ptr() + i * 2 * BLOCK * Hkv * d * 2, cap[i], n[i], T[i]]
                          for i, r in enumerate(row0)], dtype=np.int64)
    if c["kind"] == "append":
        s["k"], s["v"] = (mean + chan * normal(tokens, Hkv, d)).bfloat16(), normal(tokens, Hkv, d).bfloat16()
    else:
        s["q"] = (normal(tokens, Hkv * G, d) / chan.repeat_interleave(G, 1) * 1.5).bfloat16()
        s["o"] = torch.empty((tokens, Hkv * G, d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((tokens, Hkv * G), dtype=torch.float32, device="cuda")
        s["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    if c["kind"] == "sparse":
        s["idx"] = torch.empty((tokens, Hkv, c["n_sel"]), dtype=torch.int32, device="cuda")
    return s


# -------------------------------------------------------------------- run --
def run(s):
    return {"append": _append, "attend": _attend, "sparse": _sparse}[s["case"]["kind"]](s)


def _append(s):
    if own:
        import paper_2606_20537_amd as cap
        cap.kvb_append(s["seqs"], s["k"], s["v"])
    else:
        for g in s["groups"]:
            b0, old = divmod(g["n"] - g["T"], BLOCK)
            for side, new in enumerate((s["k"], s["v"])):
                _put(s, g, torch.cat([s["open"][g["at"], side, :old], new[g["tokens"]]], 1), side, b0)
    return {"k": s["kv"][0].view(E4M3), "v": s["kv"][1].view(E4M3), "scales": s["scales"], "bounds": s["bounds"].view(E4M3),
            "open": s["open"]}


def _attend(s):
    if own:
        import paper_2606_20537_amd as cap
        cap.kvb_attend(s["seqs"], s["q"], s["o"], kv_heads=s["case"]["Hkv"], lse=s["lse"], scale=s["scale"], workspace=s["workspace"])
        return {"o": s["o"], "lse": s["lse"]}
    o, lse = torch.empty_like(s["o"]), torch.empty_like(s["lse"])
    for g in s["groups"]:
        for a, b in _pieces(s, g):
            o[g["tokens"][:, a:b]], lse[g["tokens"][:, a:b]] = _dense(s, g, a, b)
    return {"o": o, "lse": lse}


def _sparse(s):
    c = s["case"]
    if own:
        import paper_2606_20537_amd as cap
        cap.kvb_select(s["seqs"], s["q"], s["idx"], kv_heads=c["Hkv"], first=c["first"], last=c["last"], workspace=s["workspace"])
        cap.kvb_attend(s["seqs"], s["q"], s["o"], kv_heads=c["Hkv"], lse=s["lse"], scale=s["scale"], idx=s["idx"],
                       workspace=s["workspace"])
        return {"idx": s["idx"], "o": s["o"], "lse": s["lse"]}
    idx, o, lse = (torch.empty_like(s[name]) for name in ("idx", "o", "lse"))
    for g in s["groups"]:
        x = idx[g["tokens"]] = _select(s, g)
        o[g["tokens"]], lse[g["tokens"]] = _chosen(s, g, x)
    return {"idx": idx, "o": o, "lse": lse}


def _values(s, g, side, rows):
    """Rows [0, rows) of K or V of the sequences of group g, [B, Hkv, rows, d] in 32 bits."""
    row = s["row0"][g["at"], None] + torch.arange(rows, device="cuda")
    x = s["kv"][side][row].view(E4M3).float() * s["scales"][row // BLOCK, side][..., None]
    return x.transpose(1, 2)


def _pieces(s, g):
    """The tokens of a step in pieces [a, b) whose scores fit the card."""
    T, step = g["T"], max(1, (1 << 32) // (len(g["at"]) * g["n"] * s["case"]["Hkv"] * s["case"]["G"]))
    return [(a, min(T, a + step)) for a in range(0, T, step)]


def _softmax(x, v):
    """x: scores [..., rows, keys], -inf where a key is not seen; v: [..., keys, d]."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.where(z > 0, (p @ v) / z, 0.0)
    return o, (m + z.log()).squeeze(-1)


def _dense(s, g, a, b):
    """Tokens [a, b) of the step of the sequences of group g."""
    c, B = s["case"], len(g["at"])
    pos = torch.arange(g["n"] - g["T"] + a, g["n"] - g["T"] + b, device="cuda")
    seen = g["n"] - g["T"] + b  # rows that the last of them sees
    k, v = (_values(s, g, side, seen) for side in (0, 1))
    q = s["q"][g["tokens"][:, a:b]].float().view(B, b - a, c["Hkv"], c["G"], c["d"]).permute(0, 2, 3, 1, 4)
    x = q.flatten(2, 3) @ k.transpose(2, 3) * s["scale"]  # [B, Hkv, G * tokens, rows]
    shape = (B, c["Hkv"], c["G"], b - a)
    x.view(*shape, seen).masked_fill_(torch.arange(seen, device="cuda") > pos[:, None], -math.inf)
    o, lse = _softmax(x, v)
    return o.view(*shape, -1).permute(0, 3, 1, 2, 4).flatten(2, 3).bfloat16(), lse.view(shape).permute(0, 3, 1, 2).flatten(2, 3)


def _select(s, g):
    """The blocks of each token and KV head of the sequences of group g, [B, T, Hkv, n_sel], ascending, then -1: its own
    block and those before it up to `last` in all, the first `first`, then those that score highest (ties: the lowest
    index).  A block's score is the highest that a key within its bounds could have with any of the head's queries."""
    c, B = s["case"], len(g["at"])
    nb = -(-g["n"] // BLOCK)
    blocks = s["row0"][g["at"], None] // BLOCK + torch.arange(nb, device="cuda")
    # products of bf16 and E4M3 values and their sums are exact in 64 bits: two blocks never change places by rounding
    lo, hi = s["bounds"][blocks].view(E4M3).double().permute(2, 0, 3, 4, 1)  # [B, Hkv, d, nb]
    q = s["q"][g["tokens"]].double().view(B, -1, c["Hkv"], c["G"], c["d"]).transpose(1, 2).flatten(2, 3)
    score = (q.clamp(max=0) @ lo + q.clamp(min=0) @ hi).view(B, c["Hkv"], -1, c["G"], nb).amax(3)
    score = (score * s["scales"][blocks, 0].double().transpose(1, 2)[:, :, None]).transpose(1, 2).contiguous()  # [B, T, Hkv, nb]
    block = torch.arange(nb, device="cuda")
    mine = (torch.arange(g["n"] - g["T"], g["n"], device="cuda") // BLOCK)[:, None, None]
    score = torch.where(score.isnan() | (block < c["first"]) | (block > mine - c["last"]), math.inf, score)
    # the blocks that a token has to have stand before those whose score is infinite
    order = torch.where(block > mine, -math.inf, score).sort(dim=-1, descending=True, stable=True)[1]
    must = ((order < c["first"]) | (order > mine - c["last"])) & (order <= mine)
    order = order.gather(-1, must.to(torch.uint8).sort(dim=-1, descending=True, stable=True)[1])
    idx = torch.where(order <= mine, order, nb)[..., :c["n_sel"]].sort(dim=-1)[0]
    idx = torch.nn.functional.pad(idx, (0, c["n_sel"] - idx.shape[-1]), value=nb)
    return torch.where(idx < nb, idx, -1).int()


def _chosen(s, g, idx):
    c, B = s["case"], len(g["at"])
    pos = torch.arange(g["n"] - g["T"], g["n"], device="cuda")[:, None, None]
    row = (idx.long()[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(3)  # [B, T, Hkv, keys]
    hidden = (row < 0) | (row > pos)
    row, head = row.masked_fill(hidden, 0) + s["row0"][g["at"], None, None, None], torch.arange(c["Hkv"], device="cuda")[:, None]
    k, v = (s["kv"][side].view(E4M3)[row, head].float() * s["scales"][row // BLOCK, side, head][..., None] for side in (0, 1))
    q = s["q"][g["tokens"]].float().view(B, -1, c["Hkv"], c["G"], c["d"])
    x = (q @ k.transpose(3, 4) * s["scale"]).masked_fill_(hidden[..., None, :], -math.inf)
    o, lse = _softmax(x, v)
    return o.flatten(2, 3).bfloat16(), lse.flatten(2, 3)


# ------------------------------------------------------------------- work --
def work(case):
    c = case
    n, T, Hkv, G, d = _ints(c["n"]), _ints(c["T"]), c["Hkv"], c["G"], c["d"]
    H, tokens = Hkv * G, sum(T)
    if c["kind"] == "append":
        # new rows read, their codes and those kept for the open blocks written; scales and bounds of the blocks begun
        blocks = sum(-(-m // BLOCK) - (m - t) // BLOCK for m, t in zip(n, T))
        kept = sum(min(t, m % BLOCK) for m, t in zip(n, T))
        return {"bytes": tokens * Hkv * d * (4 + 2) + kept * Hkv * d * 4 + blocks * Hkv * (8 + 2 * d), "flops": tokens * Hkv * d * 4}
    io = tokens * H * (d * 4 + 4)
    if c["kind"] == "attend":
        pairs = sum(t * m - t * (t - 1) // 2 for m, t in zip(n, T))
        return {"bytes": io + sum(n) * Hkv * d * 2 + sum(-(-m // BLOCK) for m in n) * Hkv * 8, "flops": 4 * H * d * pairs}
    nb = [-(-m // BLOCK) for m in n]
    read = sum(min(m, BLOCK * c["n_sel"]) for m in n)  # rows that one token at least has to read
    pairs = sum(t * min(m, BLOCK * c["n_sel"]) for m, t in zip(n, T))
    return {"bytes": io + tokens * Hkv * c["n_sel"] * 4 + sum(nb) * Hkv * (2 * d + 4) + read * Hkv * d * 2 + read // BLOCK * Hkv * 8,
            "flops": 4 * H * d * (sum(t * b for t, b in zip(T, nb)) + pairs)}


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    """Written from the definitions, in 64 bits, sequence by sequence and head by head."""
    s = prepare(case, seed)
    c, f64 = case, torch.float64
    if c["kind"] == "append":
        return _exact_append(s)
    n, T, row0, Hkv, G, d = _ints(c["n"]), _ints(c["T"]), s["row0"].tolist(), c["Hkv"], c["G"], c["d"]
    tokens = sum(T)
    o = torch.zeros((tokens, Hkv * G, d), dtype=f64, device="cuda")
    lse = torch.full((tokens, Hkv * G), -math.inf, dtype=f64, device="cuda")
    picked = torch.full((tokens, Hkv, c["n_sel"]), -1, dtype=torch.int32, device="cuda")
    t0 = 0
    for i in range(len(n)):
        nb, b0, r0 = -(-n[i] // BLOCK), row0[i] // BLOCK, row0[i]
        at = torch.arange(n[i], device="cuda") // BLOCK
        for h in range(Hkv):
            group = slice(h * G, (h + 1) * G)
            k, v = (s["kv"][side][r0:r0 + n[i], h].view(E4M3).to(f64) * s["scales"][b0 + at, side, h].to(f64)[:, None] for side in (0, 1))
            step = max(1, (1 << 29) // (n[i] * G))
            for a in range(0, T[i], step):
                b = min(T[i], a + step)
                pos = torch.arange(n[i] - T[i] + a, n[i] - T[i] + b, device="cuda")
                q = s["q"][t0 + a:t0 + b, group].to(f64)
                seen = torch.arange(n[i], device="cuda") <= pos[:, None]
                if c["kind"] == "sparse":
                    lo, hi = (s["bounds"][b0:b0 + nb, side, h].view(E4M3).to(f64) for side in (0, 1))
                    chosen = torch.zeros((b - a, nb), dtype=torch.bool, device="cuda")
                    for t in range(b - a):
                        upper = torch.maximum(q[t][:, None] * lo, q[t][:, None] * hi).sum(-1).amax(0) * s["scales"][b0:b0 + nb, 0, h].to(f64)
                        mine = int(pos[t]) // BLOCK
                        must = set(range(min(c["first"], mine + 1))) | set(range(max(0, mine - c["last"] + 1), mine + 1))
                        rank = upper.tolist()
                        rest = sorted((x for x in range(mine + 1) if x not in must), key=lambda x: (-rank[x], x))
                        keep = sorted(must | set(rest[:max(0, c["n_sel"] - len(must))]))
                        picked[t0 + a + t, h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
                        chosen[t, keep] = True
                    seen &= chosen[:, at]
                x = (q @ k.t()) * s["scale"]  # [T, G, n]
                x.masked_fill_(~seen[:, None], -math.inf)
                lse[t0 + a:t0 + b, group] = torch.logsumexp(x, -1)
                o[t0 + a:t0 + b, group] = torch.softmax(x, -1) @ v
        t0 += T[i]
    return {"idx": picked, "o": o, "lse": lse} if c["kind"] == "sparse" else {"o": o, "lse": lse}


def _exact_append(s):
    c, f64, row0 = s["case"], torch.float64, s["row0"].tolist()
    out = {"k": s["kv"][0].view(E4M3).to(f64), "v": s["kv"][1].view(E4M3).to(f64), "scales": s["scales"].to(f64),
           "bounds": s["bounds"].view(E4M3).to(f64), "open": s["open"].to(f64)}
    t0 = 0
    for i, (n, T) in enumerate(zip(_ints(c["n"]), _ints(c["T"]))):
        for name, side in (("k", 0), ("v", 1)):
            first = (n - T) // BLOCK * BLOCK
            rows = torch.cat([s["open"][i, side, :n - T - first], s[name][t0:t0 + T]]).to(f64)
            full = rows.shape[0] // BLOCK * BLOCK
            for part in (rows[:full].view(-1, BLOCK, c["Hkv"], c["d"]), rows[None, full:]):
                if part.numel() == 0:
                    continue
                b = (row0[i] + first) // BLOCK + (full // BLOCK if part.shape[1] < BLOCK else 0)
                scale = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 3), keepdim=True) / 448.0)))
                y = part / scale
                # nearest multiple of the spacing of E4M3 at this magnitude, ties to even
                gap = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                y = torch.round(y / gap) * gap
                out[name][b * BLOCK:b * BLOCK + y.shape[0] * y.shape[1]] = y.flatten(0, 1)
                out["scales"][b:b + y.shape[0], side] = scale[:, 0, :, 0]
                if side == 0:
                    out["bounds"][b:b + y.shape[0]] = torch.stack([y.amin(1), y.amax(1)], 1)
            if rows.shape[0] % BLOCK:
                out["open"][i, side, :rows.shape[0] % BLOCK] = rows[full:]
        t0 += T
    return out
