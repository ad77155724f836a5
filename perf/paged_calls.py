"""Times of calls over paged bf16 caches that the listed cases of more_operators.py do not have: runs of tokens (prompts,
resumed turns, drafts of many sessions), caches whose table is wider than the rows held, and rows of float32.

    python3 perf/paged_calls.py [runs] [tables] [rows]

Microseconds of a call on the GPU, the least of several replays of a graph of such calls, beside its floor: the bytes that it cannot do
without at 6.49 TB/s or its products at 1218 TFLOP/s, whichever is more."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_20537_amd as cap  # noqa: E402

BYTES, FLOPS = 6.49e6, 1.218e9  # a microsecond

# rows of a sequence, sequences, tokens of each, query heads of one of four KV heads
RUNS = [(16384, 1, 16384, 8), (8192, 1, 8192, 4), (2048, 16, 512, 4), (2048, 1, 2048, 4), (512, 1, 512, 4), (100, 64, 32, 4), (16545, 1, 161, 8),
        (2048, 32, 9, 8), (16384, 8, 4, 8)]
# the same, and KV heads
TABLES = [(200, 1, 1, 8, 4), (300, 8, 1, 8, 4), (816, 32, 1, 8, 1), (300, 8, 6, 16, 4), (816, 32, 6, 8, 4), (16385, 1, 1, 8, 4)]
# tokens, query heads, KV heads, channels
ROWS = [(16384, 32, 4, 256), (4159, 16, 4, 128), (2000, 8, 1, 256)]


def time_of(call, heavy=False):
    call()
    torch.cuda.synchronize()
    graph, n = torch.cuda.CUDAGraph(), 1 if heavy else 10
    with torch.cuda.graph(graph):
        for _ in range(n):
            call()
    best = float("inf")
    for _ in range(3 if heavy else 9):
        graph.replay()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / (2 * n))
    return best


def attention(d, n, B, T, G, Hkv, columns=0, page=64):
    """(us, floor) of B sequences of n rows, the last T of which are the call's tokens."""
    need = -(-n // page)
    pools = torch.randn((2, B * need, page, Hkv, d), dtype=torch.bfloat16, device="cuda")
    table = torch.full((B, max(columns, need)), -1, dtype=torch.int32, device="cuda")
    table[:, :need] = torch.randperm(B * need, device="cuda").view(B, need)
    cache = cap.kvp_cache(pools[0], pools[1], table)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    tok0 = torch.arange(B + 1, dtype=torch.int32, device="cuda") * T
    q = torch.randn((B * T, Hkv * G, d), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    space = torch.empty(max(16, cap.kvp_attend_workspace_bytes(cache, B * T, Hkv * G)), dtype=torch.uint8, device="cuda")
    pairs = B * sum(range(n - T + 1, n + 1))
    us = time_of(lambda: cap.kvp_attend(cache, lens, q, o, scale=d ** -0.5, tok0=tok0, workspace=space), pairs > 1 << 25)
    return us, max((4 * B * n * Hkv * d + 4 * q.numel()) / BYTES, 4 * pairs * Hkv * G * d / FLOPS)


def rotation(tokens, Hq, Hkv, d, dtype):
    q, k = (torch.randn((tokens, h, d), device="cuda").to(dtype) for h in (Hq, Hkv))
    w, pos = torch.ones(d, device="cuda").to(dtype), torch.arange(tokens, dtype=torch.int32, device="cuda")
    rule = cap.qk_rule(cap.qk_freqs(1e6, 64).cuda(), wq=w, wk=w, eps=1e-6)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    return time_of(lambda: cap.qk_norm_rope(rule, q, k, qo, ko, pos=pos)), 2 * (q.numel() + k.numel()) * q.element_size() / BYTES


def main(parts):
    if "runs" in parts:
        for n, B, T, G in RUNS:
            text = ["%d: %8.1f (floor %7.1f)" % (d, *attention(d, n, B, T, G, 4)) for d in (64, 128, 256)]
            print("%2d x %5d rows, %5d tokens, %2d heads on 4, channels " % (B, n, T, 4 * G), ",  ".join(text), flush=True)
    if "tables" in parts:
        for n, B, T, G, Hkv in TABLES:
            for d in (64, 128, 256):
                text = ["%6d rows %6.1f" % (rows, attention(d, n, B, T, G, Hkv, rows // 64)[0]) for rows in (n, 1024, 16384, 131072) if rows >= n]
                print("%2d x %5d rows, %d tokens, %2d heads on %d of %3d, a table of " % (B, n, T, G * Hkv, Hkv, d), ", ".join(text), flush=True)
    if "rows" in parts:
        for tokens, Hq, Hkv, d in ROWS:
            text = ["%s %6.1f (floor %6.1f)" % (str(t)[6:], *rotation(tokens, Hq, Hkv, d, t)) for t in (torch.bfloat16, torch.float32)]
            print("%5d tokens, %d + %d heads of %d, norm and rotation: " % (tokens, Hq, Hkv, d), ",  ".join(text), flush=True)


if __name__ == "__main__":
    main(sys.argv[1:] or ["runs", "tables", "rows"])
