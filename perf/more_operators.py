"""The operators of a full-attention layer over paged bf16 caches, as programs
call them: the calls, their plain forms, and their results in 64 bits.

A cache is a pool of pages of K and one of V, [pages, page rows, KV heads, d],
and a table that names the pages of each sequence in order (-1: none).  A step
covers a batch of sequences of their own lengths n, each with T tokens at
positions [n - T, n); q, k, v and o are packed [sum of T, heads, d].

  rotate   root-mean-square norm of each head of q and k, then the rotation of
           its first channels by angles that are sums over the axes of a
           token's position
  append   T new rows of K and V enter the pages; with a rule, q and k are
           normed and rotated on the way
  attend   causal attention of the T newest tokens over the pages

``listed`` gives the fixed cases, ``draw`` more of the same ranges, ``prepare``
what the program holds before the call, ``run`` one pass, ``work`` the bytes and
operations that it cannot do without, ``exact`` its results in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
BASE = 1.0e6  # of the frequencies


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # one decode token of each of the 32 robot environments: 8 + 1 heads of 256
        _rotate("rotate_step_32_envs", tokens=32, Hq=8, Hkv=1, d=256, rot=64),
        # one layer of the 48-layer stack over its 16k prefix; the projection gives
        # each query head and its output gate side by side, then K and V
        _rotate("rotate_16k", tokens=16384, Hq=32, Hkv=4, d=256, rot=64, fused=True, w_add=1.0),
        # a video of 4159 patches: time, height and width turn channels of their own
        _rotate("rotate_video", tokens=4159, Hq=16, Hkv=4, d=128, rot=128, axes=3),
        # fp32 tokens of a short suffix about position 2^20, neighbouring channels
        # paired, no norm
        _rotate("rotate_far_f32", tokens=257, Hq=4, Hkv=4, d=64, rot=64, pairs=True, norm=False, dtype="f32", start=1 << 20),
        # one token of each of the 32 robot environments enters its cache, its q
        # and k normed and rotated in the same pass
        _append("append_step_32_envs", n="816*32", T="1*32", Hkv=1, G=8, d=256, page=64, rot=64),
        # the whole 16k prefix of one layer of the 48-layer stack
        _append("append_16k", n="16384", T="16384", Hkv=4, G=8, d=256, page=64, rot=64),
        # rows that are ready as they are: suffixes of four sessions of the 8-layer
        # stack, begun and ended inside small pages
        _append("append_ragged", n="2111,8191,4159,67", T="161,2047,33,67", Hkv=4, G=4, d=128, page=16, rot=0),
        # decode, the smallest model: 200 rows, 4 KV heads of 64, small pages
        _attend("decode_200_d64", n="200", T="1", Hkv=4, G=2, d=64, page=16),
        # decode of the 32 robot environments
        _attend("decode_32_envs", n="816*32", T="1*32", Hkv=1, G=8, d=256, page=64),
        # decode of one session of the 48-layer stack behind its 16k prefix
        _attend("decode_16k", n="16385", T="1", Hkv=4, G=8, d=256, page=64),
        # decode of four sessions, from a fresh one to a long one, and one that waits
        _attend("decode_ragged_131k", n="131072,16449,2111,1,700", T="1*4,0", Hkv=4, G=8, d=256, page=64),
        # three tokens (one and two drafts) of each of 64 sessions of the 8-layer
        # stack that see the last 1000 rows
        _attend("drafts_64_window", n="8191*16,2111*32,130*16", T="3*64", Hkv=4, G=4, d=128, page=32, window=1000),
    ]


def _rotate(name, tokens, Hq, Hkv, d, rot, axes=1, norm=True, w_add=0.0, pairs=False, dtype="bf16", fused=False, start=0):
    return {"name": name, "kind": "rotate", "tokens": tokens, "Hq": Hq, "Hkv": Hkv, "d": d, "rot": rot, "axes": axes, "norm": norm,
            "w_add": w_add, "pairs": pairs, "dtype": dtype, "fused": fused, "start": start}


def _append(name, n, T, Hkv, G, d, page, rot, w_add=0.0, pairs=False):
    """n and T: a number for each sequence, as text ("816*32": 32 times 816).  rot = 0: no rule."""
    return {"name": name, "kind": "append", "n": n, "T": T, "Hkv": Hkv, "G": G, "d": d, "page": page, "rot": rot, "axes": 1,
            "norm": True, "w_add": w_add, "pairs": pairs}


def _attend(name, n, T, Hkv, G, d, page, window=0):
    return {"name": name, "kind": "attend", "n": n, "T": T, "Hkv": Hkv, "G": G, "d": d, "page": page, "window": window}


def _ints(text):
    return [int(a.split("*")[0]) for a in text.split(",") for _ in range(int(a.split("*")[1]) if "*" in a else 1)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: 1 to 16384 tokens of 1 to 8 KV heads with 1 to 16 query heads to each, 1 to 64 sequences of 1 to
    131072 rows, pages of 16 to 256 rows."""
    kind = rng.choice(["rotate", "append", "attend", "attend"])
    Hkv, G = rng.choice([1, 2, 3, 4, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    page = rng.choice([16, 32, 48, 64, 64, 128, 256])
    if kind == "rotate":
        d = rng.choice([64, 80, 96, 128, 192, 256])
        most = 16384 * 36 * 256 // ((Hkv * G + Hkv) * d)
        c = _rotate("", _log_int(rng, 1, min(16384, most)), Hkv * G, Hkv, d, 16 * rng.randint(1, d // 16), axes=rng.randint(1, 3),
                    norm=rng.random() < 0.75, w_add=rng.choice([0.0, 1.0]), pairs=rng.random() < 0.4,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), fused=rng.random() < 0.5, start=rng.choice([0, 0, 16385, 1 << 20]))
        if c["dtype"] == "f32":
            c["tokens"] = (c["tokens"] + 1) // 2
    elif kind == "append":
        d = rng.choice([64, 128, 256])
        B = _log_int(rng, 1, 64)
        most = 16384 * 40 * 256 // ((G + 2) * Hkv * d)
        T = [_log_int(rng, 1, max(1, min(16384, most) // B)) if rng.random() < 0.6 else 1 for _ in range(B)]
        n = [t + _log_int(rng, 1, 4096) - 1 for t in T]
        c = _append("", ",".join(map(str, n)), ",".join(map(str, T)), Hkv, G, d, page,
                    16 * rng.randint(1, d // 16) if rng.random() < 0.7 else 0, rng.choice([0.0, 1.0]), rng.random() < 0.4)
    else:
        d = rng.choice([64, 128, 256])
        B = _log_int(rng, 1, 64)
        T = [1] * B if rng.random() < 0.6 else [rng.randint(1, 6) for _ in range(B)]
        n = [max(t, _log_int(rng, 1, 131072)) for t in T]
        rows = 150000 * 1024 // (Hkv * d)
        while sum(n) > rows:
            n = [max(t, m // 2) for t, m in zip(T, n)]
        c = _attend("", ",".join(map(str, n)), ",".join(map(str, T)), Hkv, G, d, page,
                    _log_int(rng, 16, 8192) if rng.random() < 0.3 else 0)
    del c["name"]
    return c


# ---------------------------------------------------------------- prepare --
def _frequencies(rot, axes):
    """Radians per position of each axis and pair: one axis turns a pair, the axes take turns."""
    i = torch.arange(rot // 2, device="cuda")
    f = torch.exp(-2.0 * i.double() / max(1, rot) * math.log(BASE))
    return torch.where(i % axes == torch.arange(axes, device="cuda")[:, None], f, 0.0)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 29)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    s = {"case": c}
    if c["kind"] == "rotate":
        tokens, Hq, Hkv = c["tokens"], c["Hq"], c["Hkv"]
    else:
        n, T = _ints(c["n"]), _ints(c["T"])
        tokens, Hkv, Hq = sum(T), c["Hkv"], c["Hkv"] * c["G"]
    d = c["d"]
    if c["kind"] != "attend" and c.get("rot"):
        dtype = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
        s["freqs"] = _frequencies(c["rot"], c["axes"])
        s["wq"], s["wk"] = ((1.0 - c["w_add"] + 0.2 * normal(d)).to(dtype) if c["norm"] else None for _ in range(2))
    if c["kind"] == "rotate":
        # heads are of mixed size, a few channels of large values
        size = torch.exp(normal(1, Hq + Hkv, 1) + 0.5 * normal(1, 1, d))
        if c["fused"]:  # [query head, gate] by query head, then K, then V
            x = normal(tokens, 2 * Hq + 2 * Hkv, d)
            x[:, :2 * Hq:2] *= size[:, :Hq]
            x[:, 2 * Hq:2 * Hq + Hkv] *= size[:, Hq:]
            x = x.to(dtype)
            s["q"], s["k"] = x[:, :2 * Hq:2], x[:, 2 * Hq:2 * Hq + Hkv]
        else:
            s["q"], s["k"] = (normal(tokens, Hq, d) * size[:, :Hq]).to(dtype), (normal(tokens, Hkv, d) * size[:, Hq:]).to(dtype)
        i = torch.arange(tokens, device="cuda")  # frames of 24 x 36 patches
        s["pos"] = (torch.stack([i] if c["axes"] == 1 else [i // 864, i // 36 % 24, i % 36][:c["axes"]], 1) + c["start"]).int()
        s["q_out"], s["k_out"] = (torch.empty((tokens, h, d), dtype=dtype, device="cuda") for h in (Hq, Hkv))
    else:
        page = c["page"]
        s["n"], s["T"] = n, T
        # sequences of the same lengths, which the plain form takes together
        first = [sum(T[:i]) for i in range(len(T))]
        s["groups"] = [{"n": m, "T": t, "at": torch.tensor(at, device="cuda"), "tokens": torch.tensor([first[i] for i in at], device="cuda")[:, None]
                        + torch.arange(t, device="cuda")}
                       for m, t, at in ((m, t, [i for i in range(len(n)) if (n[i], T[i]) == (m, t)]) for m, t in dict.fromkeys(zip(n, T))) if t]
        need = [-(-m // page) for m in n]
        held = sum(need)
        pages = held + 5
        order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32).tolist()
        table = torch.full((len(n), max(need) + 1), -1, dtype=torch.int32)
        for i, m in enumerate(need):
            table[i, :m] = torch.tensor(order[sum(need[:i]):sum(need[:i]) + m], dtype=torch.int32)
        s["table"] = table.cuda()
        s["lens"] = torch.tensor(n, dtype=torch.int32, device="cuda")
        s["tok0"] = torch.tensor(first + [tokens], dtype=torch.int32, device="cuda")
        # keys have a few channels of large values and an offset, as models' keys do; values are of mixed size by head
        chan = torch.exp(0.5 * normal(1, 1, Hkv, d))
        mean = 0.5 * normal(1, 1, Hkv, d) * chan
        s["k_pages"] = (mean + chan * normal(pages, page, Hkv, d)).bfloat16()
        s["v_pages"] = (torch.exp(normal(1, 1, Hkv, 1)) * normal(pages, page, Hkv, d)).bfloat16()
        if c["kind"] == "append":
            s["k"], s["v"] = (mean[0] + chan[0] * normal(tokens, Hkv, d)).bfloat16(), normal(tokens, Hkv, d).bfloat16()
            s["q"], s["q_out"] = (normal(tokens, Hq, d).bfloat16(), torch.empty((tokens, Hq, d), dtype=torch.bfloat16, device="cuda")) if c["rot"] else (None, None)
        else:
            s["scale"] = 1.0 / math.sqrt(d)
            s["q"] = (normal(tokens, Hq, d) / chan[0].repeat_interleave(c["G"], 1) * 1.5).bfloat16()
            s["o"] = torch.empty((tokens, Hq, d), dtype=torch.bfloat16, device="cuda")
            s["lse"] = torch.empty((tokens, Hq), dtype=torch.float32, device="cuda")
    if own:  # the handles that a program makes once and keeps
        import paper_2606_20537_amd as cap
        if "freqs" in s:
            s["rule"] = cap.qk_rule(s["freqs"], wq=s["wq"], wk=s["wk"], eps=EPS if c["norm"] else None, w_add=c["w_add"], pairs=c["pairs"])
        if "table" in s:
            s["cache"] = cap.kvp_cache(s["k_pages"], s["v_pages"], s["table"])
        if c["kind"] == "attend":
            s["workspace"] = torch.empty(cap.kvp_attend_workspace_bytes(s["cache"], tokens, Hq), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------- run --
def run(s):
    return {"rotate": _run_rotate, "append": _run_append, "attend": _run_attend}[s["case"]["kind"]](s)


def _run_rotate(s):
    if own:
        import paper_2606_20537_amd as cap
        cap.qk_norm_rope(s["rule"], s["q"], s["k"], s["q_out"], s["k_out"], pos=s["pos"])
        return {"q": s["q_out"], "k": s["k_out"]}
    return {"q": _turned(s, s["q"], s["wq"], s["pos"]), "k": _turned(s, s["k"], s["wk"], s["pos"])}


def _run_append(s):
    c = s["case"]
    if own:
        import paper_2606_20537_amd as cap
        if c["rot"]:
            cap.kvp_append(s["cache"], s["lens"], s["k"], s["v"], tok0=s["tok0"], rule=s["rule"], q=s["q"], q_out=s["q_out"])
        else:
            cap.kvp_append(s["cache"], s["lens"], s["k"], s["v"], tok0=s["tok0"])
        return {"k": s["k_pages"], "v": s["v_pages"], "q": s["q_out"]} if c["rot"] else {"k": s["k_pages"], "v": s["v_pages"]}
    q, k, pos, row = s["q"], s["k"], torch.empty((len(s["k"]), 1), dtype=torch.int32, device="cuda"), torch.empty(len(s["k"]), dtype=torch.int64, device="cuda")
    for g in s["groups"]:
        p = torch.arange(g["n"] - g["T"], g["n"], device="cuda")
        pos[g["tokens"], 0] = p.int().expand(g["tokens"].shape)
        row[g["tokens"]] = _rows(s, g, p)
    if c["rot"]:
        q, k = _turned(s, q, s["wq"], pos), _turned(s, k, s["wk"], pos)
    s["k_pages"].flatten(0, 1)[row] = k
    s["v_pages"].flatten(0, 1)[row] = s["v"]
    return {"k": s["k_pages"], "v": s["v_pages"], "q": q} if c["rot"] else {"k": s["k_pages"], "v": s["v_pages"]}


def _run_attend(s):
    c = s["case"]
    if own:
        import paper_2606_20537_amd as cap
        cap.kvp_attend(s["cache"], s["lens"], s["q"], s["o"], scale=s["scale"], tok0=s["tok0"], window=c["window"], lse=s["lse"],
                       workspace=s["workspace"])
        return {"o": s["o"], "lse": s["lse"]}
    o, lse = torch.empty_like(s["o"]), torch.empty_like(s["lse"])
    for g in s["groups"]:
        o[g["tokens"]], lse[g["tokens"]] = _seen(s, g)
    return {"o": o, "lse": lse}


def _turned(s, x, w, pos):
    """x [tokens, heads, d] normed and rotated, rounded once."""
    c, y, rot = s["case"], x.float(), s["case"]["rot"]
    if c["norm"]:
        y = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt() * (c["w_add"] + w.float())
    angle = (pos.double()[:, :, None] * s["freqs"]).sum(1)[:, None]  # far positions need 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = (y[..., :rot:2], y[..., 1:rot:2]) if c["pairs"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(2) if c["pairs"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _rows(s, g, at):
    """Rows of the pools that hold the rows `at` of the sequences of group g, [B, rows]."""
    page = s["case"]["page"]
    return s["table"][g["at"]][:, at // page].long() * page + at % page


def _seen(s, g):
    """Attention of the tokens of the sequences of group g."""
    c, B, n, T = s["case"], len(g["at"]), g["n"], g["T"]
    pos = torch.arange(n - T, n, device="cuda")
    lo = max(0, n - T - c["window"] + 1) if c["window"] else 0
    at = torch.arange(lo, n, device="cuda")
    row = _rows(s, g, at)
    k, v = (s[name].flatten(0, 1)[row].float().transpose(1, 2) for name in ("k_pages", "v_pages"))  # [B, Hkv, rows, d]
    q = s["q"][g["tokens"]].float().view(B, T, c["Hkv"], c["G"], c["d"]).permute(0, 2, 3, 1, 4)
    x = (q.flatten(2, 3) @ k.transpose(2, 3).contiguous() * s["scale"]).view(B, c["Hkv"], c["G"], T, n - lo)
    hidden = at > pos[:, None]
    if c["window"]:
        hidden |= at <= pos[:, None] - c["window"]
    x = x.masked_fill_(hidden, -math.inf).flatten(2, 3)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o, lse = (p @ v) / z, (m + z.log()).squeeze(-1)
    o, lse = o.view(B, c["Hkv"], c["G"], T, -1), lse.view(B, c["Hkv"], c["G"], T)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3).bfloat16(), lse.permute(0, 3, 1, 2).flatten(2, 3)


# ------------------------------------------------------------------- work --
def work(case):
    c = case
    d = c["d"]
    if c["kind"] == "rotate":
        size = 4 if c["dtype"] == "f32" else 2
        values = c["tokens"] * (c["Hq"] + c["Hkv"]) * d
        return {"bytes": 2 * size * values + 4 * c["tokens"] * c["axes"] + (2 * size * d if c["norm"] else 0) + 4 * c["rot"] * c["axes"],
                "flops": values * (4 if c["norm"] else 0) + values * c["rot"] // d * 3}
    n, T, Hkv, G, page = _ints(c["n"]), _ints(c["T"]), c["Hkv"], c["G"], c["page"]
    tokens = sum(T)
    index = 4 * (2 * len(n) + 1)
    if c["kind"] == "append":
        values = tokens * Hkv * d * (G + 2 if c["rot"] else 2)
        index += 4 * sum(-(-m // page) - (m - t) // page for m, t in zip(n, T))
        return {"bytes": 4 * values + index, "flops": tokens * Hkv * d * (G + 1) * 7 if c["rot"] else 0}
    w = c["window"]
    first = [max(0, m - t - w + 1) if w else 0 for m, t in zip(n, T)]
    rows = sum(m - f for m, t, f in zip(n, T, first) if t)
    pairs = sum(min(m - i, w) if w else m - i for m, t in zip(n, T) for i in range(t))
    index += 4 * sum(-(-m // page) - f // page for m, t, f in zip(n, T, first) if t)
    return {"bytes": rows * Hkv * d * 4 + tokens * Hkv * G * (4 * d + 4) + index, "flops": 4 * Hkv * G * d * pairs}


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    """Written from the definitions, in 64 bits, sequence by sequence."""
    s = prepare(case, seed)
    c = case
    if c["kind"] == "rotate":
        return {"q": _exact_turn(s, s["q"], s["wq"], s["pos"].double()), "k": _exact_turn(s, s["k"], s["wk"], s["pos"].double())}
    if c["kind"] == "append":
        out = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
        new = {"k": s["k"].double(), "v": s["v"].double()}
        if c["rot"]:
            pos = torch.cat([torch.arange(n - t, n, device="cuda") for n, t in zip(s["n"], s["T"])]).double()[:, None]
            new["k"], out["q"] = _exact_turn(s, s["k"], s["wk"], pos), _exact_turn(s, s["q"], s["wq"], pos)
        t0 = 0
        for i, (n, t) in enumerate(zip(s["n"], s["T"])):
            at = torch.arange(n - t, n, device="cuda")
            of = s["table"][i].long()[at // c["page"]]
            for name in ("k", "v"):
                out[name][of, at % c["page"]] = new[name][t0:t0 + t]
            t0 += t
        return out
    f64, G, tokens = torch.float64, c["G"], sum(s["T"])
    o = torch.zeros((tokens, c["Hkv"] * G, c["d"]), dtype=f64, device="cuda")
    lse = torch.zeros((tokens, c["Hkv"] * G), dtype=f64, device="cuda")
    t0 = 0
    for i, (n, T) in enumerate(zip(s["n"], s["T"])):
        if T:
            of = s["table"][i, :-(-n // c["page"])].long()
            for h in range(c["Hkv"]):
                k, v = (s[name][of, :, h].flatten(0, 1)[:n].to(f64) for name in ("k_pages", "v_pages"))
                for t in range(T):
                    last = n - T + t
                    lo = max(0, last - c["window"] + 1) if c["window"] else 0
                    x = s["q"][t0 + t, h * G:(h + 1) * G].to(f64) @ k[lo:last + 1].t() * s["scale"]
                    lse[t0 + t, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
                    o[t0 + t, h * G:(h + 1) * G] = torch.softmax(x, -1) @ v[lo:last + 1]
        t0 += T
    return {"o": o, "lse": lse}


def _exact_turn(s, x, w, pos):
    """Each pair of channels as a complex number, times e^(i angle)."""
    c, rot = s["case"], s["case"]["rot"]
    y = x.double()
    if c["norm"]:
        y = y / torch.sqrt(torch.mean(y * y, -1, keepdim=True) + EPS) * (c["w_add"] + w.double())
    angle = pos @ s["freqs"]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + rot // 2)
    z = torch.complex(y[..., a], y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y
