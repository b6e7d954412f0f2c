"""The operators that work on a whole paged cache at once, as they are measured: the attention of a chunk of new tokens
("chunk"), the same with the weight that every cached token receives ("weigh"), the heaviest tokens kept in a smaller cache
("keep"), and a decode step's attention over the blocks that a cheap score selects ("sparse").

`run` computes each in a plain form (elementary torch operations, 32 bits, one rounding at the end; the scores that select
blocks in 64) or, where `own` is set, calls the library.
"""
import math

import numpy as np
import torch

own = False

DIM = 128                     # elements of a head row
PAGE = 64                     # token slots of a page, tokens of a block


# ---- cases -------------------------------------------------------------------------------------------------------

def listed():
    return [
        # five drafted tokens of one sequence, checked in one go: latency
        dict(op="chunk", name="chunk draft", layers=1, batch=1, tokens=5, context=256, q_heads=8, kv_heads=2),
        # four drafted tokens of each of 32 sequences, four layers of long caches
        dict(op="chunk", name="chunk draft batch 32", layers=4, batch=32, tokens=4, context=8192, q_heads=28, kv_heads=4),
        # the next turn of four conversations, lengths that end inside pages and tiles
        dict(op="chunk", name="chunk next turn", layers=2, batch=4, tokens=511, context=1000, q_heads=32, kv_heads=8),
        # a piece of a long document, one layer
        dict(op="chunk", name="chunk long document", layers=1, batch=1, tokens=4096, context=28671, q_heads=40, kv_heads=8),
        # what the newest token looks at, one sequence
        dict(op="weigh", name="weigh last token", layers=1, batch=1, tokens=1, context=511, q_heads=8, kv_heads=2),
        # what the last 64 tokens of long prompts look at, eight layers
        dict(op="weigh", name="weigh window", layers=8, batch=4, tokens=64, context=8128, q_heads=28, kv_heads=4),
        # whole prompts, every token's weight over all later ones
        dict(op="weigh", name="weigh prompts", layers=1, batch=2, tokens=4096, context=0, q_heads=32, kv_heads=8),
        # one sequence, one layer, cut to a fraction
        dict(op="keep", name="keep few", layers=1, batch=1, tokens=700, keep=250, recent=32, initial=4, q_heads=28, kv_heads=4),
        # 32 sequences, eight layers, a quarter stays
        dict(op="keep", name="keep batch 32", layers=8, batch=32, tokens=8192, keep=2048, recent=128, initial=0, q_heads=28, kv_heads=4),
        # a short cache, a few blocks
        dict(op="sparse", name="sparse short", layers=1, batch=1, tokens=1030, blocks=8, index=False, q_heads=8, kv_heads=2),
        # the first step after prompts were loaded: the blocks' bounds are made too
        dict(op="sparse", name="sparse first step", layers=4, batch=8, tokens=16384, blocks=32, index=True, q_heads=32, kv_heads=8),
        # a step of 16 sequences over long documents
        dict(op="sparse", name="sparse long documents", layers=1, batch=16, tokens=131071, blocks=64, index=False, q_heads=40, kv_heads=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    q_heads, kv_heads = rng.choice([(8, 2), (28, 4), (32, 8), (40, 8), (6, 6), (9, 3), (16, 2), (12, 2)])
    op = rng.choice(["chunk", "chunk", "weigh", "keep", "sparse"])
    layers, batch = _log(rng, 1, 16), _log(rng, 1, 32)
    case = dict(op=op, layers=layers, batch=batch, q_heads=q_heads, kv_heads=kv_heads)
    if op in ("chunk", "weigh"):
        case["tokens"] = rng.choice([1, _log(rng, 1, 16), _log(rng, 16, 4096), _log(rng, 16, 512)])
        case["context"] = rng.choice([0, _log(rng, 1, 32768), _log(rng, 256, 16384)])
    elif op == "keep":
        case["tokens"] = _log(rng, 64, 32768)
        case["recent"] = _log(rng, 1, max(1, case["tokens"] // 4))
        case["initial"] = rng.choice([0, 0, 4, 17])
        least = case["recent"] + case["initial"] + 1
        case["keep"] = rng.choice([_log(rng, least, max(least, case["tokens"])), _log(rng, least, max(least, case["tokens"] // 2))])
    else:
        case["tokens"] = _log(rng, 1, 131072)
        case["blocks"] = _log(rng, 1, 128)
        case["index"] = rng.random() < 0.3

    def too_much():
        units, n = case["layers"] * case["batch"] * kv_heads, case["tokens"] + case.get("context", 0)
        return units * n > 8.4e6 or work(case)["flops"] > 2.4e12 * (0.25 if op == "weigh" else 1.0)

    while too_much():                                        # fewer sequences, then fewer layers, then a shorter chunk
        which = "batch" if case["batch"] > 1 else "layers" if case["layers"] > 1 else "tokens"
        case[which] = max(1, case[which] // 2)
    return case


# ---- what a user's program has in hand ----------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _shape(case):
    return case["layers"], case["batch"], case["q_heads"], case["kv_heads"], case["tokens"] + case.get("context", 0)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    L, B, Hq, Hkv, n = _shape(case)
    T = case["tokens"] if case["op"] in ("chunk", "weigh") else 1

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)

    k, v = normal(L, B, Hkv, n, DIM), normal(L, B, Hkv, n, DIM)
    if case["op"] == "keep":
        # what tokens have received over time: a few a lot, most of them little
        weights = torch.exp(2 * torch.randn(L * B * Hkv, n, generator=g, device="cuda"))
    else:
        # the queries as a projection leaves them, beside the chunk's keys and values
        s["q"] = normal(L, B, T, Hq + 2 * Hkv, DIM)[..., :Hq, :]
        # a few keys that a query attends to strongly (+4 on the scaled logit), in some heads many of one kind
        first = s["q"][:, :, 0].float().reshape(L, B, Hkv, Hq // Hkv, DIM)[:, :, :, 0]
        first = first * (4 * math.sqrt(DIM) / first.square().sum(-1, keepdim=True))
        k[:, :, :, ::97] += first.unsqueeze(3).to(k.dtype)
    if not own:
        s["k"], s["v"] = k, v
        if case["op"] == "keep":
            s["weights"] = weights
        elif case["op"] == "sparse":
            full = n // PAGE - (n % PAGE == 0)               # blocks before the newest
            rows = k[..., :full * PAGE, :].unflatten(3, (full, PAGE))
            s["high"], s["low"] = rows.amax(4), rows.amin(4)
        return s
    from paper_2506_15969_b200 import binding
    if case["op"] == "keep":
        S, R = case["initial"], case["recent"]
        s["cache"] = binding.Engine(L, Hq, Hkv, DIM, n + R + S + 1, 1, 2.0, batch=B, n_recent=R, n_initial=S, weights=True)
        s["cache"].set_score_mode(binding.SCORE_WEIGHT)
        s["cache"].prefill(k, v)
        s["cache"].state_views()["weights"][:, :n] = weights
        s["small"] = binding.Engine(L, Hq, Hkv, DIM, case["keep"] + 1, 1, 2.0, batch=B, weights=True)
        s["views"] = s["small"].state_views()
        return s
    s["cache"] = binding.Engine(L, Hq, Hkv, DIM, n + 1, 1, 2.0, batch=B, weights=case["op"] == "weigh")
    s["cache"].prefill(k, v)
    if case["op"] == "sparse":
        s["q"] = s["q"][:, :, 0].contiguous()
        s["selected"] = torch.empty(L * B * Hkv, case["blocks"], dtype=torch.int32, device="cuda")
        s["cache"].index_blocks()
    s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    s["views"] = s["cache"].state_views()
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def _chunk(s):
    """Rows of the last tokens over everything up to themselves, some units (layer, sequence, KV head) at a time."""
    case = s["case"]
    L, B, Hq, Hkv, n = _shape(case)
    T, G, U = case["tokens"], Hq // Hkv, L * B * Hkv
    q = s["q"].unflatten(3, (Hkv, G)).permute(0, 1, 3, 2, 4, 5).reshape(U, T * G, DIM)
    k, v = s["k"].view(U, n, DIM), s["v"].view(U, n, DIM)
    sees = torch.arange(n, device="cuda") <= n - T + torch.arange(T, device="cuda").repeat_interleave(G)[:, None]
    out = torch.empty(U, T * G, DIM, dtype=torch.bfloat16, device="cuda")
    weights = torch.empty(U, n, device="cuda")
    some = max(1, int(1e9 // (T * G * n)))
    for u in range(0, U, some):
        i = slice(u, u + some)
        x = (q[i].float() / math.sqrt(DIM)) @ k[i].float().mT
        x = torch.where(sees, x, -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        total = x.sum(-1, keepdim=True)
        out[i] = ((x @ v[i].float()) / total).to(out.dtype)
        if case["op"] == "weigh":
            weights[i] = (x / total).sum(1) / G
    out = out.view(L, B, Hkv, T, G, DIM).transpose(2, 3).reshape(L, B, T, Hq, DIM)
    return {"out": out, "weights": weights} if case["op"] == "weigh" else {"out": out}


def _to_pages(rows, pages, half):
    """rows [units, n, 128] into slots 0 .. n-1: page i / 64, row r = i % 64, 16-byte chunk c at c ^ (r & 7)."""
    i = torch.arange(rows.shape[1], device=rows.device)
    chunk = torch.arange(DIM // 8, device=rows.device) ^ (i % PAGE & 7)[:, None]
    pages[:, i // PAGE, half, i % PAGE] = rows.unflatten(-1, (DIM // 8, 8))[:, i[:, None], chunk]


def _keep(s):
    case = s["case"]
    L, B, _, Hkv, n = _shape(case)
    S, R, U, keep = case["initial"], case["recent"], L * B * Hkv, min(case["keep"], n)
    pages = torch.zeros(U, (case["keep"] + 2 + PAGE - 1) // PAGE, 2, PAGE, DIM // 8, 8, dtype=torch.bfloat16, device="cuda")
    w = s["weights"]
    at = torch.arange(n, device="cuda").expand(U, n)
    if keep < n:
        # the first and the newest stay, of the others the heaviest; of equals the newer
        order = w[:, S:n - R].flip(1).sort(dim=1, descending=True, stable=True).indices[:, :keep - S - R]
        middle = (n - R - 1 - order).sort(1).values
        at = torch.cat((at[:, :S], middle, at[:, n - R:]), 1)
    some = max(1, int(4e8 // (keep * DIM)))
    for u in range(0, U, some):
        i = slice(u, u + some)
        for half, x in enumerate((s["k"], s["v"])):
            _to_pages(x.view(U, n, DIM)[i].gather(1, at[i, :, None].expand(-1, -1, DIM)), pages[i], half)
    return {"pages": pages.view(-1, 2, PAGE, DIM), "pos": at.to(torch.int32), "weights": w.gather(1, at)}


def _sparse(s):
    case = s["case"]
    L, B, Hq, Hkv, n = _shape(case)
    G, U, last = Hq // Hkv, L * B * Hkv, (n - 1) // PAGE
    k, v = s["k"].view(U, n, DIM), s["v"].view(U, n, DIM)
    q = s["q"].reshape(U, G, DIM)
    if case["index"]:
        rows = k[:, :last * PAGE].unflatten(1, (last, PAGE))
        high, low = rows.amax(2), rows.amin(2)
    else:
        high, low = s["high"].view(U, last, DIM), s["low"].view(U, last, DIM)
    # the largest sum over the heads of the logits that a key between the block's bounds can have; close ones in 64 bits
    q64 = q.double()
    up, down = q64.clamp(min=0).sum(1), q64.clamp(max=0).sum(1)
    blocks = min(case["blocks"], last + 1)
    chosen = torch.full((U, case["blocks"]), -1, dtype=torch.int32, device="cuda")
    some = max(1, int(2e8 // (max(last, 1) * DIM)))
    for u in range(0, U, some):
        i = slice(u, u + some)
        score = (high[i].double() @ up[i, :, None] + low[i].double() @ down[i, :, None]).squeeze(-1)
        best = score.sort(dim=1, descending=True, stable=True).indices[:, :blocks - 1]     # of equals the older
        chosen[i, :blocks - 1] = best.sort(1).values.to(torch.int32)
    chosen[:, blocks - 1] = last                             # the newest block always
    at = (chosen[:, :blocks, None].long() * PAGE + torch.arange(PAGE, device="cuda")).flatten(1)
    out = torch.empty(U, G, DIM, dtype=torch.bfloat16, device="cuda")
    some = max(1, int(2e8 // (blocks * PAGE * DIM)))
    for u in range(0, U, some):
        i = slice(u, u + some)
        rows = at[i].clamp(max=n - 1)[..., None].expand(-1, -1, DIM)
        x = (q[i].float() / math.sqrt(DIM)) @ k[i].gather(1, rows).float().mT
        x = torch.where((at[i] < n)[:, None], x, -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        out[i] = ((x @ v[i].gather(1, rows).float()) / x.sum(-1, keepdim=True)).to(out.dtype)
    done = {"out": out.view(L, B, Hq, DIM), "selected": chosen}
    if case["index"]:
        done["bounds"] = torch.stack((high, low), 2)         # [units, blocks, 2, 128]
    return done


def run(s):
    case = s["case"]
    n = _shape(case)[4]
    if not own:
        return _keep(s) if case["op"] == "keep" else _sparse(s) if case["op"] == "sparse" else _chunk(s)
    if case["op"] == "chunk":
        s["cache"].attend_chunk(s["q"], s["out"])
        return {"out": s["out"]}
    if case["op"] == "weigh":
        from paper_2506_15969_b200 import binding
        s["cache"].attend_chunk(s["q"], s["out"], weights=binding.WEIGHTS_SET)
        return {"out": s["out"], "weights": s["views"]["weights"][:, :n]}
    if case["op"] == "keep":
        keep = min(case["keep"], n)
        s["small"].reset()                                   # the small cache is used again for the next prompts
        s["cache"].evict_to(case["keep"], s["small"])
        return {"pages": s["views"]["pages"], "pos": s["views"]["pos"][:, :keep], "weights": s["views"]["weights"][:, :keep]}
    if case["index"]:
        s["cache"].index_blocks(0)
    s["cache"].attend_sparse(s["q"], s["out"], case["blocks"], s["selected"])
    done = {"out": s["out"], "selected": s["selected"]}
    if case["index"]:
        done["bounds"] = s["cache"].block_bounds()[:, :(n - 1) // PAGE]
    return done


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    L, B, Hq, Hkv, n = _shape(case)
    units, G = L * B * Hkv, Hq // Hkv
    if case["op"] in ("chunk", "weigh"):
        T = case["tokens"]
        pairs = L * B * Hq * (T * (n - T) + T * (T + 1) // 2)          # (query row, key) pairs
        rows = L * B * Hq * T
        if case["op"] == "chunk":
            return {"bytes": 512 * units * n + 512 * rows, "flops": 4 * DIM * pairs}
        # a row's weights need its sum: logits before and after it is known
        return {"bytes": 512 * units * n + 512 * rows + 4 * units * n, "flops": 6 * DIM * pairs}
    if case["op"] == "keep":
        keep = min(case["keep"], n)
        # the weights; of the kept tokens K, V, (TS, MRI), position and weight, read and written
        return {"bytes": units * (4 * (n - keep) + keep * 2 * (512 + 16)), "flops": units * n}
    last, blocks = (n - 1) // PAGE, min(case["blocks"], (n + PAGE - 1) // PAGE)
    index = 256 * last * PAGE + 512 * last if case["index"] else 512 * last
    return {"bytes": units * (index + 512 * min(n, blocks * PAGE) + 512 * G + 4 * case["blocks"]),
            "flops": units * (2 * 2 * DIM * last + 4 * DIM * G * min(n, blocks * PAGE))}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------

def _exact_attention(q, k, v, mask):
    """One unit: q [rows, 128], k and v [n, 128], mask [rows, n] of what a row sees; also the probabilities."""
    x = (q.double() @ k.double().T).div_(math.sqrt(DIM)).masked_fill_(~mask, -math.inf)
    p = torch.softmax(x, -1)
    return p @ v.double(), p


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    L, B, Hq, Hkv, n = _shape(case)
    G, T = Hq // Hkv, case["tokens"]
    if case["op"] == "keep":
        # unit by unit: candidates in the order of the weights, of equals the newer first
        S, R, keep = case["initial"], case["recent"], min(case["keep"], n)
        at = np.tile(np.arange(n), (L * B * Hkv, 1))
        if keep < n:
            place = np.arange(S, n - R)
            for u, row in enumerate(s["weights"].cpu().numpy()):
                stays = place[np.lexsort((-place, -row[S:n - R]))][:keep - S - R]
                at[u, :keep] = np.concatenate((np.arange(S), np.sort(stays), np.arange(n - R, n)))
        at = torch.tensor(at[:, :keep], device="cuda")
        unit = torch.arange(at.shape[0], device="cuda")[:, None]
        pages = torch.zeros(at.shape[0], (case["keep"] + 2 + PAGE - 1) // PAGE, 2, PAGE, DIM // 8, 8, dtype=torch.float64, device="cuda")
        for half, x in enumerate((s["k"], s["v"])):
            rows = x.flatten(0, 2)[unit, at].view(*at.shape, DIM // 8, 8)
            for r in range(min(8, keep)):                    # the slots j with j % 8 = r
                j = torch.arange(r, keep, 8, device="cuda")
                for c in range(DIM // 8):
                    pages[:, j // PAGE, half, j % PAGE, c ^ r] = rows[:, j, c].double()
        return {"pages": pages.view(-1, 2, PAGE, DIM), "pos": at.to(torch.int32), "weights": s["weights"].double()[unit, at]}
    if case["op"] in ("chunk", "weigh"):
        out = torch.empty(L, B, T, Hq, DIM, dtype=torch.float64, device="cuda")
        weights = torch.zeros(L, B, Hkv, n, dtype=torch.float64, device="cuda")
        some = max(1, int(2e8 // (G * n)))                   # rows at a time
        for l in range(L):
            for b in range(B):
                for h in range(Hkv):
                    for i in range(0, T, some):
                        t = min(some, T - i)
                        q = s["q"][l, b, i:i + t, h * G:(h + 1) * G].reshape(t * G, DIM)
                        mask = torch.ones(t, n, dtype=torch.bool, device="cuda").tril(n - T + i)
                        o, p = _exact_attention(q, s["k"][l, b, h], s["v"][l, b, h], mask.repeat_interleave(G, 0))
                        out[l, b, i:i + t, h * G:(h + 1) * G] = o.view(t, G, DIM)
                        weights[l, b, h] += p.sum(0) / G
        return {"out": out, "weights": weights.view(-1, n)} if case["op"] == "weigh" else {"out": out}
    last = (n - 1) // PAGE
    blocks = min(case["blocks"], last + 1)
    out = torch.empty(L, B, Hq, DIM, dtype=torch.float64, device="cuda")
    chosen = torch.full((L, B, Hkv, case["blocks"]), -1, dtype=torch.int32, device="cuda")
    bounds = torch.empty(L, B, Hkv, last, 2, DIM, dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):
            for h in range(Hkv):
                k, q = s["k"][l, b, h], s["q"][l, b, 0, h * G:(h + 1) * G]
                for x, f in ((0, torch.amax), (1, torch.amin)):
                    bounds[l, b, h, :, x] = f(k[:last * PAGE].view(last, PAGE, DIM).double(), 1)
                # the larger of the two products in every dimension, head by head
                score = sum(torch.maximum(bounds[l, b, h, :, 0] * head, bounds[l, b, h, :, 1] * head).sum(-1) for head in q.double())
                best = torch.argsort(-score, stable=True)[:blocks - 1].tolist()
                seen = torch.zeros(n, dtype=torch.bool, device="cuda")
                for j, block in enumerate(sorted(best) + [last]):
                    chosen[l, b, h, j] = block
                    seen[block * PAGE:(block + 1) * PAGE] = True
                i = seen.nonzero().squeeze(1)
                out[l, b, h * G:(h + 1) * G] = _exact_attention(q, k[i], s["v"][l, b, h][i], seen[i].expand(G, -1))[0]
    done = {"out": out, "selected": chosen.flatten(0, 2)}
    if case["index"]:
        done["bounds"] = bounds.flatten(0, 2)
    return done
