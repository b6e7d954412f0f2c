"""The operators around the paged cache, as they are measured: head norms with the position rotation ("rope"), the
append of projected keys and values to the pages ("append"), and the attention of a batch that shares prefixes ("attend").

`run` computes each in a plain form (elementary torch operations, 32 bits, one rounding at the end) or, where `own` is
set, calls the library.
"""
import math

import torch

own = False

DIM = 128                     # elements of a head row
PAGE = 64                     # token slots of a page
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases -------------------------------------------------------------------------------------------------------

def listed():
    rope = dict(op="rope", interleaved=False, pairs=64, norm=True, first=0, dtype="bf16", out="same")
    append = dict(op="append", interleaved=False, pairs=64, norm=True, dtype="bf16")
    return [
        # one token of one sequence in one layer: nothing but latency
        dict(rope, name="rope one token", layers=1, batch=1, tokens=1, q_heads=8, kv_heads=2),
        # a decode step of 32 sequences, 28 layers in one call
        dict(rope, name="rope step batch 32", layers=28, batch=32, tokens=1, q_heads=28, kv_heads=4, first=8192),
        # a chunk of a long document: half precision, a quarter of the dimensions turn, far positions, no norm
        dict(rope, name="rope chunk fp16 partial", layers=1, batch=1, tokens=4097, q_heads=28, kv_heads=4, dtype="fp16",
             out="bf16", interleaved=True, pairs=16, norm=False, first=1000003),
        # whole prompts of a layer
        dict(rope, name="rope long prompts", layers=1, batch=2, tokens=16384, q_heads=40, kv_heads=8),
        # one token of one sequence in one layer
        dict(append, name="append one token", layers=1, batch=1, tokens=1, q_heads=8, kv_heads=2),
        # the new tokens of a decode step, 48 layers and 32 sequences in one call
        dict(append, name="append step batch 32", layers=48, batch=32, tokens=1, q_heads=40, kv_heads=8),
        # prompts that end inside a page, projections left in 32 bits
        dict(append, name="append prompts fp32", layers=4, batch=4, tokens=511, q_heads=28, kv_heads=4, dtype="fp32",
             interleaved=True),
        # prompts of a batch of 16, eight layers
        dict(append, name="append prompts", layers=8, batch=16, tokens=1024, q_heads=32, kv_heads=8),
        # four samples of a short prompt, just begun
        dict(op="attend", name="attend short prefix", layers=1, batch=4, prefixes=1, q_heads=8, kv_heads=2, prefix=256, tokens=1),
        # two prompts, sixteen samples of each, all layers; half a thousand tokens into their answers
        dict(op="attend", name="attend two prefixes", layers=28, batch=32, prefixes=2, q_heads=28, kv_heads=4, prefix=2048, tokens=512),
        # a long document that sixteen questions share, one layer; lengths that end inside a page
        dict(op="attend", name="attend long prefix", layers=1, batch=16, prefixes=1, q_heads=32, kv_heads=8, prefix=65521, tokens=130),
        # many samples of one prompt: more query rows than the prefix's bytes cost
        dict(op="attend", name="attend wide batch", layers=4, batch=128, prefixes=1, q_heads=40, kv_heads=8, prefix=8192, tokens=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    q_heads, kv_heads = rng.choice([(8, 2), (28, 4), (32, 8), (40, 8), (6, 6), (9, 3), (16, 2), (12, 2)])
    op = rng.choice(["rope", "append", "attend", "attend"])
    layers, batch = _log(rng, 1, 48), _log(rng, 1, 128)
    if op == "attend":
        prefixes = rng.choice([1, 1, 2, 3, 4])
        batch = prefixes * max(1, batch // prefixes)
        prefix, tokens = _log(rng, 1, 65536), rng.choice([0, _log(rng, 1, 2048), _log(rng, 1, 256)])
        # no more query rows times keys, and no more own tokens, than the largest listed case has
        rows = batch * q_heads
        layers = max(1, min(layers, int(1.6e8 // (rows * (prefix + tokens))), int(1.7e6 // (batch * kv_heads * max(tokens, 1))),
                            int(5e5 // (prefixes * kv_heads * prefix))))
        while layers * rows * (prefix + tokens) > 1.6e8 and prefix > 1:
            prefix = max(1, prefix // 2)
        return dict(op=op, layers=layers, batch=batch, prefixes=prefixes, q_heads=q_heads, kv_heads=kv_heads, prefix=prefix, tokens=tokens)
    tokens = rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 16384)])
    heads = q_heads + 2 * kv_heads
    while layers * batch * tokens * heads > 1.4e6:
        layers, batch, tokens = (layers // 2, batch, tokens) if layers > 1 else (1, batch // 2, tokens) if batch > 1 else (1, 1, tokens // 2)
    case = dict(op=op, layers=layers, batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, interleaved=rng.random() < 0.4,
                pairs=rng.choice([64, 64, 32, 16, 8, 0]), norm=rng.random() < 0.7, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if not case["pairs"]:
        case["norm"] = True
    if op == "rope":
        case["first"] = rng.choice([0, _log(rng, 1, 4000000)])
        case["out"] = rng.choice(["same", "bf16"])
    return case


# ---- what a user's program has in hand ----------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inv_freq(pairs):
    return [1e6 ** (-j / pairs) for j in range(pairs)]       # radians per position


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    L, B, Hq, Hkv, n = case["layers"], case["batch"], case["q_heads"], case["kv_heads"], case["tokens"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    if case["op"] == "attend":
        Pb, N = case["prefixes"], case["prefix"]
        s["q"] = normal(L, B, Hq, DIM)
        kp, vp = normal(L, Pb, Hkv, N, DIM), normal(L, Pb, Hkv, N, DIM)
        ko, vo = normal(L, B, Hkv, n, DIM), normal(L, B, Hkv, n, DIM)
        # a few keys that some query attends to strongly (+4 on the scaled logit)
        first = s["q"].view(L, B, Hkv, Hq // Hkv, DIM)[:, :, :, 0].float()
        first = first * (4 * math.sqrt(DIM) / first.square().sum(-1, keepdim=True))
        kp[:, :, :, ::97] += first[:, :: B // Pb].unsqueeze(3).to(kp.dtype)
        ko[:, :, :, ::89] += first.unsqueeze(3).to(ko.dtype)
        s.update(kp=kp, vp=vp, ko=ko, vo=vo)
        if own:
            from paper_2506_15969_b200 import binding
            # a cache with the prompts and one with the samples' own tokens, room for a few more; nothing is evicted
            s["prefix"] = binding.Engine(L, Hq, Hkv, DIM, N + 1, 1, 2.0, batch=Pb)
            s["prefix"].prefill(kp, vp)
            s["cache"] = binding.Engine(L, Hq, Hkv, DIM, n + 2, 1, 2.0, batch=B)
            s["cache"].attach_prefix(s["prefix"])
            if n:
                s["cache"].prefill(ko, vo)
            s["out"] = torch.empty_like(s["q"])
            s["views"] = s["cache"].state_views()
        return s

    # one projection gives the rows of the queries, keys and values, token by token; heads differ in size
    heads = Hq + 2 * Hkv
    qkv = normal(L, B, n, heads, DIM, dtype=TYPES[case["dtype"]])
    qkv *= torch.exp(torch.randn(heads, 1, generator=g, device="cuda")).to(qkv.dtype)
    s["q"], s["k"], s["v"] = qkv[..., :Hq, :], qkv[..., Hq:Hq + Hkv, :], qkv[..., Hq + Hkv:, :]
    if case["norm"]:
        s["qw"], s["kw"] = (torch.rand(L, DIM, generator=g, device="cuda") + 0.5 for _ in range(2))
    pages = (n + 2 + PAGE - 1) // PAGE
    if case["op"] == "rope":
        to = TYPES[case["dtype"] if case["out"] == "same" else case["out"]]
        s["to"] = to
        s["first"] = case["first"]
    if own:
        from paper_2506_15969_b200 import binding
        s["cache"] = binding.Engine(L, Hq, Hkv, DIM, n + 1 if case["op"] == "append" else 2, 1, 2.0, batch=B)
        if case["pairs"]:
            s["cache"].set_rope(_inv_freq(case["pairs"]), interleaved=case["interleaved"])
        if case["norm"]:
            s["cache"].set_head_norm(s["qw"], s["kw"], 1e-6)
        if case["op"] == "rope":
            s["q_out"] = torch.empty(L, B, n, Hq, DIM, dtype=to, device="cuda")
            s["k_out"] = torch.empty(L, B, n, Hkv, DIM, dtype=to, device="cuda")
        else:
            s["views"] = s["cache"].state_views()
    elif case["op"] == "append":
        units = L * B * Hkv
        s["pages"] = torch.zeros(units, pages, 2, PAGE, DIM // 8, 8, dtype=torch.bfloat16, device="cuda")
        s["pos"] = torch.zeros(units, pages * PAGE, dtype=torch.int32, device="cuda")
        s["ts_mri"] = torch.zeros(units, pages * PAGE, 2, dtype=torch.int32, device="cuda")
    if case["pairs"]:
        s["inv_freq"] = torch.tensor(_inv_freq(case["pairs"]), dtype=torch.float64, device="cuda")
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def _turned(x, weight, s, first):
    """Norm and rotation of head rows x [layers, batch, tokens, heads, 128], in 32 bits."""
    case, x = s["case"], x.float()
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight[:, None, None, None, :]
    if not case["pairs"]:
        return x
    p = case["pairs"]
    where = torch.arange(first, first + x.shape[2], device=x.device, dtype=torch.float64)
    angle = where[:, None] * s["inv_freq"]                   # far positions: 64 bits
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    t, rest = x[..., :2 * p], x[..., 2 * p:]
    a, b = (t[..., 0::2], t[..., 1::2]) if case["interleaved"] else (t[..., :p], t[..., p:])
    u, w = a * cos - b * sin, b * cos + a * sin
    t = torch.stack((u, w), -1).flatten(-2) if case["interleaved"] else torch.cat((u, w), -1)
    return torch.cat((t, rest), -1)


def _to_pages(rows, pages, half):
    """rows [units, n, 128] into slots 0 .. n-1: page i / 64, row r = i % 64, 16-byte chunk c at c ^ (r & 7)."""
    i = torch.arange(rows.shape[1], device=rows.device)
    chunk = torch.arange(DIM // 8, device=rows.device) ^ (i % PAGE & 7)[:, None]
    pages[:, i // PAGE, half, i % PAGE] = rows.unflatten(-1, (DIM // 8, 8))[:, i[:, None], chunk]


def _attend(s):
    case = s["case"]
    L, B, Hq, Hkv, Pb = (case[k] for k in ("layers", "batch", "q_heads", "kv_heads", "prefixes"))
    R, G, N, n = B // Pb, Hq // Hkv, case["prefix"], case["tokens"]
    q = s["q"].float().view(L, Pb, R, Hkv, G, DIM) / math.sqrt(DIM)
    # the prefix once for the R sequences that share it
    q = q.transpose(2, 3)                                                      # [L, Pb, Hkv, R, G, DIM]
    x = q.flatten(3, 4) @ s["kp"].float().transpose(-1, -2)                    # [L, Pb, Hkv, R * G, N]
    # every sequence's own tokens
    ko, vo = (s[k].float().view(L, Pb, R, Hkv, n, DIM).transpose(2, 3) for k in ("ko", "vo"))
    y = q @ ko.transpose(-1, -2)                                               # [L, Pb, Hkv, R, G, n]
    top = x.amax(-1).unflatten(-1, (R, G))
    if n:
        top = torch.maximum(top, y.amax(-1))
    x = torch.exp(x - top.flatten(-2).unsqueeze(-1))
    y = torch.exp(y - top.unsqueeze(-1))
    total = x.sum(-1).unflatten(-1, (R, G)) + y.sum(-1)
    out = (x @ s["vp"].float()).unflatten(-2, (R, G)) + y @ vo
    out = (out / total.unsqueeze(-1)).transpose(2, 3).reshape(L, B, Hq, DIM).to(s["q"].dtype)
    if not n:
        return {"out": out}
    pbar = (y / total.unsqueeze(-1)).mean(-2).transpose(2, 3)
    return {"out": out, "pbar": pbar.reshape(L * B * Hkv, n)}


def run(s):
    case = s["case"]
    n = case["tokens"]
    if case["op"] == "rope":
        if own:
            s["cache"].norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], first_position=s["first"])
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": _turned(s["q"], s.get("qw"), s, s["first"]).to(s["to"]),
                "k": _turned(s["k"], s.get("kw"), s, s["first"]).to(s["to"])}
    if case["op"] == "append":
        if own:
            s["cache"].reset()                               # the cache is used again for the next prompts
            s["cache"].append(s["k"], s["v"])
            v = s["views"]
            return {"pages": v["pages"], "pos": v["pos"][:, :n], "ts_mri": v["ts_mri"][:, :n]}
        rows = _turned(s["k"], s.get("kw"), s, 0).to(torch.bfloat16), s["v"].float().to(torch.bfloat16)
        for half in range(2):
            _to_pages(rows[half].transpose(2, 3).flatten(0, 2), s["pages"], half)
        s["pos"][:, :n] = torch.arange(n, device="cuda", dtype=torch.int32)
        s["ts_mri"][:, :n] = 0
        return {"pages": s["pages"].view(-1, 2, PAGE, DIM), "pos": s["pos"][:, :n], "ts_mri": s["ts_mri"][:, :n]}
    if own:
        s["cache"].attend(s["q"], s["out"])
        if not n:
            return {"out": s["out"]}
        return {"out": s["out"], "pbar": s["views"]["pbar"][:, :n]}
    return _attend(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    L, B, Hq, Hkv, n = (case[k] for k in ("layers", "batch", "q_heads", "kv_heads", "tokens"))
    if case["op"] == "attend":
        Pb, N = case["prefixes"], case["prefix"]
        return {"bytes": 512 * L * Hkv * (Pb * N + B * n) + 4 * L * B * Hkv * n + 2 * 256 * L * B * Hq,
                "flops": 4 * DIM * L * B * Hq * (N + n)}
    size = TYPES[case["dtype"]].itemsize
    tokens = L * B * n
    if case["op"] == "rope":
        rows = tokens * (Hq + Hkv)
        return {"bytes": rows * DIM * (size + (2 if case["out"] == "bf16" else size)), "flops": 10 * rows * DIM}
    # K and V rows read and written in 16 bits; position, TS and MRI written
    return {"bytes": tokens * Hkv * (2 * DIM * (size + 2) + 12), "flops": 10 * tokens * Hkv * DIM}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------

def _exact_rows(x, weight, case, first):
    """One (layer, sequence) at a time; the rotation as a product of complex numbers."""
    x = x.to(torch.float64).clone()
    L, B, n, H, _ = x.shape
    p = case["pairs"]
    if case["norm"]:
        for l in range(L):
            ms = (x[l] ** 2).sum(-1) / DIM + 1e-6
            x[l] = x[l] / torch.sqrt(ms)[..., None] * weight[l].double()
    if p:
        where = torch.arange(first, first + n, device=x.device, dtype=torch.float64)
        freq = torch.tensor(_inv_freq(p), dtype=torch.float64, device=x.device)
        turn = torch.polar(torch.ones(n, p, dtype=torch.float64, device=x.device), torch.outer(where, freq))
        for l in range(L):
            t = x[l][..., : 2 * p]
            z = torch.view_as_complex(t.unflatten(-1, (p, 2)).contiguous()) if case["interleaved"] else torch.complex(t[..., :p].contiguous(), t[..., p:].contiguous())
            z = z * turn[:, None, :]
            x[l][..., : 2 * p] = torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat((z.real, z.imag), -1)
    return x


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    L, B, Hq, Hkv, n = (case[k] for k in ("layers", "batch", "q_heads", "kv_heads", "tokens"))
    if case["op"] == "rope":
        return {"q": _exact_rows(s["q"], s.get("qw"), case, case["first"]), "k": _exact_rows(s["k"], s.get("kw"), case, case["first"])}
    if case["op"] == "append":
        k, v = _exact_rows(s["k"], s.get("kw"), case, 0), s["v"]
        pages = torch.zeros(s["pages"].shape, dtype=torch.float64, device="cuda")
        for half, rows in enumerate((k, v)):
            rows = rows.double().permute(0, 1, 3, 2, 4).reshape(L * B * Hkv, n, DIM // 8, 8)
            for c in range(DIM // 8):
                for r in range(min(8, n)):                   # the slots i with i % 8 = r
                    i = torch.arange(r, n, 8, device="cuda")
                    pages[:, i // PAGE, half, i % PAGE, c ^ r] = rows[:, i, c]
        return {"pages": pages.view(-1, 2, PAGE, DIM), "pos": None, "ts_mri": None}
    Pb, G, N = case["prefixes"], Hq // Hkv, case["prefix"]
    R = B // Pb
    out = torch.empty(L, B, Hq, DIM, dtype=torch.float64, device="cuda")
    pbar = torch.empty(L, B, Hkv, n, dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):                                   # a sequence's keys are its prefix's, then its own
            k = torch.cat((s["kp"][l, b // R], s["ko"][l, b]), 1).double()
            v = torch.cat((s["vp"][l, b // R], s["vo"][l, b]), 1).double()
            q = s["q"][l, b].double().view(Hkv, G, DIM)
            p = torch.softmax(torch.bmm(q, k.mT) / math.sqrt(DIM), -1)
            out[l, b] = torch.bmm(p, v).reshape(Hq, DIM)
            pbar[l, b] = p[..., N:].sum(1) / G
    return {"out": out, "pbar": pbar.view(L * B * Hkv, n)} if n else {"out": out}
