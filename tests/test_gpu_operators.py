"""The operators around the cache against plain 64-bit forms: head norms with the position rotation, the append of
projected rows to the pages, attention over a shared prefix; and a run of them together, as a server uses them.

Tolerances.  A rounding to a type is off by at most eps / 2 of the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).  Besides it:
* rows: the norm's factor carries about 10 roundings of 2^-24 (a sum of 128 squares in 12 levels, halved by the root; rsqrt 2
  ulp), the rotation's factors about 6 (an angle below half a turn in fp32 is 2^-22 off, sin / cos 2 ulp), products and the
  final fma 4: below 2^-19 of |y_a| + |y_b| for the two elements of a pair.
* attention: a logit is a sum of 128 exact products in fp32, off by at most 128 * 2^-23 of the sum of their
  magnitudes, which is below 50 here after scaling, typically 2^-18 of it; weights enter the second product with 16 bits, exp2 with 22.
  Both sides of the softmax move with it: 2^-13 of sum_i p_i |v_i| for an output, 2^-13 of a probability.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import lazyev_oracle as orc
from paper_2506_15969_b200 import binding

pytestmark = pytest.mark.gpu

D = 128
TYPES = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def f64(x):
    return x.detach().to("cpu", torch.float64).numpy()


def freqs(pairs, base=1e4):
    return [base ** (-j / max(pairs, 1)) for j in range(pairs)]


def engine(layers, q_heads, kv_heads, batch, tokens, window=1, threshold=2.0, **kw):
    """An engine that holds `tokens` tokens and a few more per unit and evicts nothing on its own account."""
    e = binding.Engine(layers, q_heads, kv_heads, D, tokens + window + 1, window, threshold, batch=batch, **kw)
    e.set_auto_evict(False)
    return e


def rows_ref(x, weight, eps, positions, inv_freq, interleaved=False, amplitude=1.0):
    """oracle.norm_rope over [layers, batch, tokens, heads, 128]; positions [batch][tokens]; also |y_a| + |y_b| per element."""
    x = f64(x)
    out, size = np.empty_like(x), np.empty_like(x)
    pairs = len(inv_freq)
    for l in range(x.shape[0]):
        w = None if weight is None else f64(weight[l])
        for b in range(x.shape[1]):
            out[l, b] = orc.norm_rope(x[l, b], w, eps, positions[b], inv_freq, interleaved, amplitude)
            y = np.abs(orc.norm_rope(x[l, b], w, eps, positions[b], []))
            mate = np.zeros_like(y)
            for j in range(pairs):
                a, c = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
                mate[..., a], mate[..., c] = y[..., c], y[..., a]
            size[l, b] = (y + mate) * max(1.0, abs(amplitude))
    return out, size


def assert_rows(got, ref, size, dtype):
    err = np.abs(f64(got) - ref)
    tol = TYPES[dtype] * np.abs(ref) + 2.0 ** -19 * size + (2.0 ** -25 if dtype == torch.float16 else 1e-38)
    assert np.all(err <= tol), f"worst {np.max(err / tol)} of the tolerance"


# ---- norm and rotation -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("layers,batch,tokens,hq,hkv,pairs,interleaved,norm,din,dout", [
    (1, 1, 1, 8, 2, 64, False, True, torch.bfloat16, torch.bfloat16),
    (2, 3, 1, 7, 1, 64, True, True, torch.bfloat16, torch.bfloat16),
    (1, 2, 5, 9, 3, 24, False, True, torch.float16, torch.float16),
    (3, 1, 17, 28, 4, 8, False, False, torch.float32, torch.bfloat16),
    (1, 1, 33, 40, 8, 8, True, True, torch.float32, torch.float32),
    (2, 2, 64, 6, 6, 32, True, False, torch.bfloat16, torch.float32),
    (1, 5, 3, 32, 8, 0, False, True, torch.float16, torch.bfloat16),
    (1, 1, 129, 1, 1, 40, False, True, torch.bfloat16, torch.float16),
    (2, 3, 2, 12, 2, 56, True, True, torch.float32, torch.float16),
])
def test_norm_rope_against_64_bits(layers, batch, tokens, hq, hkv, pairs, interleaved, norm, din, dout):
    g = gen(hash((layers, batch, tokens, pairs)) & 0xFFFF)
    e = engine(layers, hq, hkv, batch, 1)
    qkv = randn(g, layers, batch, tokens, hq + 2 * hkv, D) .to(din)           # a fused projection; the rows are views of it
    q, k = qkv[..., :hq, :], qkv[..., hq:hq + hkv, :]
    f = freqs(pairs)
    e.set_rope(f, interleaved=interleaved, amplitude=1.25)
    qw = kw = None
    if norm:
        qw, kw = (torch.rand(layers, D, generator=g, device="cuda") + 0.5 for _ in range(2))
        e.set_head_norm(qw, kw, 1e-5)
    qo = torch.empty(layers, batch, tokens, hq, D, dtype=dout, device="cuda")
    ko = torch.empty(layers, batch, tokens, hkv, D, dtype=dout, device="cuda")
    e.norm_rope(q, k, qo, ko, first_position=77)
    e.synchronize()
    at = [77 + np.arange(tokens)] * batch
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        ref, size = rows_ref(x, w, 1e-5, at, f, interleaved, 1.25)
        assert_rows(got, ref, size, dout)


@pytest.mark.parametrize("tokens,hq,hkv,pairs,interleaved,dtype", [
    (1301, 10, 5, 64, False, torch.bfloat16),    # a warp per token, rows that do not fill a stage
    (650, 21, 3, 16, True, torch.float16),
    (1200, 3, 3, 40, False, torch.float32),
    (40, 41, 41, 64, False, torch.bfloat16),     # more KV heads than a warp keeps pages of
    (700, 35, 35, 32, True, torch.float32),
])
def test_norm_rope_and_append_of_many_tokens(tokens, hq, hkv, pairs, interleaved, dtype):
    g = gen(tokens)
    L, B = 1, 2
    e = engine(L, hq, hkv, B, tokens)
    e.set_page_table(np.random.RandomState(1).permutation(e.info().units * e.info().pages_per_unit))
    qkv = randn(g, L, B, tokens, hq + 2 * hkv, D).to(dtype)
    q, k, v = qkv[..., :hq, :], qkv[..., hq:hq + hkv, :], qkv[..., hq + hkv:, :]
    f = freqs(pairs)
    e.set_rope(f, interleaved=interleaved)
    w = torch.rand(L, D, generator=g, device="cuda") + 0.5
    e.set_head_norm(w, w, 1e-6)
    pos = torch.randint(0, 100000, (B, tokens), generator=g, device="cuda", dtype=torch.int32)
    at = [p.cpu().numpy() for p in pos]
    ref_q, ref_k = rows_ref(q, w, 1e-6, at, f, interleaved), rows_ref(k, w, 1e-6, at, f, interleaved)
    for out in (torch.bfloat16, dtype):
        qo, ko = torch.empty(q.shape, dtype=out, device="cuda"), torch.empty(k.shape, dtype=out, device="cuda")
        e.norm_rope(q, k, qo, ko, positions=pos)
        q1, k1 = torch.empty_like(qo), torch.empty_like(ko)
        e.norm_rope(q, None, q1, None, positions=pos)
        e.norm_rope(None, k, None, k1, positions=pos)
        e.synchronize()
        assert_rows(qo, *ref_q, out)
        assert_rows(ko, *ref_k, out)
        assert torch.equal(qo, q1) and torch.equal(ko, k1)
    e.append(k, v, positions=pos)
    d = e.dump_state(kv=True)
    gk = orc.bf16_bits_to_f64(d["k"]).reshape(L, B, hkv, tokens, D).transpose(0, 1, 3, 2, 4)
    assert_rows(torch.from_numpy(gk.copy()), *ref_k, torch.bfloat16)
    gv = orc.bf16_bits_to_f64(d["v"]).reshape(L, B, hkv, tokens, D).transpose(0, 1, 3, 2, 4)
    assert np.array_equal(gv, f64(v.to(torch.bfloat16)))
    assert np.array_equal(d["pos"][0], np.arange(tokens))               # the cache's own order, whatever the keys turn by
    # in place, queries and keys in one call
    e.norm_rope(q, k, q, k, positions=pos)
    e.synchronize()
    assert_rows(q, *ref_q, dtype)
    assert_rows(k, *ref_k, dtype)


def test_rows_more_than_four_gigabytes_apart():
    """Strides and pages behind 32-bit offsets: two sequences whose rows lie 4.8 GB apart, pages at the end of a pool of 9 GB."""
    g = gen(6)
    Hq, Hkv, T = 4, 2, 70
    flat = torch.empty(2 ** 31 + 2 ** 28, dtype=torch.bfloat16, device="cuda")
    n = T * (Hq + 2 * Hkv) * D
    x = flat.as_strided((1, 2, T, Hq + 2 * Hkv, D), (0, flat.numel() - n, (Hq + 2 * Hkv) * D, D, 1))
    x.copy_(randn(g, *x.shape))
    e = binding.Engine(1, Hq, Hkv, D, 2 ** 22, 64, 2.0, batch=2)
    inf = e.info()
    assert inf.units * inf.pages_per_unit * 32768 > 2 ** 32
    e.set_page_table(np.arange(inf.units * inf.pages_per_unit)[::-1].copy())
    f = freqs(64)
    e.set_rope(f)
    qo = torch.empty(1, 2, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    e.norm_rope(x[..., :Hq, :], None, qo, None)
    e.append(x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :])
    d = e.dump_state(kv=True)
    assert_rows(qo, *rows_ref(x[..., :Hq, :], None, 0, [np.arange(T)] * 2, f), torch.bfloat16)
    ref, size = rows_ref(x[..., Hq:Hq + Hkv, :], None, 0, [np.arange(T)] * 2, f)
    gk = orc.bf16_bits_to_f64(d["k"]).reshape(1, 2, Hkv, T, D).transpose(0, 1, 3, 2, 4)
    assert_rows(torch.from_numpy(gk.copy()), ref, size, torch.bfloat16)
    gv = orc.bf16_bits_to_f64(d["v"]).reshape(1, 2, Hkv, T, D).transpose(0, 1, 3, 2, 4)
    assert np.array_equal(gv, f64(x[..., Hq + Hkv:, :]))


def test_norm_rope_positions_views_and_in_place():
    g = gen(5)
    L, B, T, Hq, Hkv = 2, 3, 6, 5, 5
    e = engine(L, Hq, Hkv, B, 1)
    f = freqs(64, 1e6)
    e.set_rope(f)
    w = torch.rand(L, D, generator=g, device="cuda") + 0.5
    e.set_head_norm(w, None, 1e-6)                                      # queries only
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789]] * B, dtype=torch.int32, device="cuda")
    pos[1] = pos[1].flip(0)
    base = randn(g, B, Hq, L, T, D)                                     # another order of the dimensions
    q = base.permute(2, 0, 3, 1, 4)
    k = randn(g, L, 1, T, Hkv, D).expand(L, B, T, Hkv, D)               # one row for all sequences (stride 0)
    ko = torch.empty(T, Hkv, B, L, D, dtype=torch.bfloat16, device="cuda").permute(3, 2, 0, 1, 4)
    at = [p.cpu().numpy().astype(np.int64) for p in pos]
    ref_q, size_q = rows_ref(q, w, 1e-6, at, f)
    ref_k, size_k = rows_ref(k, None, 1e-6, at, f)
    e.norm_rope(q, k, q, ko, positions=pos)                             # queries in place
    e.synchronize()
    assert_rows(q, ref_q, size_q, torch.bfloat16)
    assert_rows(ko, ref_k, size_k, torch.bfloat16)
    # one side alone, and a single token without its dimension
    q1 = randn(g, L, B, 1, Hq, D)
    o1 = torch.empty_like(q1)
    e.norm_rope(q1, None, o1, None, first_position=9)
    k1 = torch.empty(L, B, 1, Hkv, D, dtype=torch.bfloat16, device="cuda")
    e.norm_rope(None, q1, None, k1, first_position=9)
    e.synchronize()
    assert_rows(o1, *rows_ref(q1, w, 1e-6, [[9]] * B, f), torch.bfloat16)
    assert_rows(k1, *rows_ref(q1, None, 1e-6, [[9]] * B, f), torch.bfloat16)


def test_row_calls_refuse_bad_arguments():
    e = engine(1, 8, 2, 2, 10)
    lib, h = binding.lib(), e._h
    x = torch.zeros(1, 2, 4, 8, D, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 2, 4, 2, D, dtype=torch.bfloat16, device="cuda")

    class Rows(C.Structure):             # lazyev_rows_t
        _fields_ = [("data", C.c_void_p), ("dtype", C.c_int), ("stride_layer", C.c_longlong), ("stride_batch", C.c_longlong),
                    ("stride_token", C.c_longlong), ("stride_head", C.c_longlong)]

    def rows(t, **kw):
        r = Rows(t.data_ptr(), binding.BF16, *t.stride()[:4])
        for name, v in kw.items():
            setattr(r, name, v)
        return C.byref(r)

    def refused(rc, word):
        assert rc == binding.EINVAL and word in lib.lazyev_last_error(h).decode(), lib.lazyev_last_error(h)

    call = lambda q, qo, n=4: lib.lazyev_norm_rope(h, q, None, n, None, 0, qo, None)      # noqa: E731
    assert call(rows(x), rows(x)) == binding.OK
    refused(call(rows(x), rows(x), 0), "no rows")
    refused(lib.lazyev_norm_rope(h, None, None, 4, None, 0, None, None), "no rows")
    refused(call(rows(x), None), "q_out")
    refused(call(rows(x, data=x.data_ptr() + 2), rows(x)), "16-byte aligned")
    refused(call(rows(x, stride_head=132), rows(x)), "multiples of 16 bytes")
    refused(call(rows(x, dtype=5), rows(x)), "type")
    refused(call(rows(x), rows(x, stride_batch=0)), "overlap")
    refused(call(rows(x), rows(x, data=None)), "null")
    refused(lib.lazyev_append(h, rows(k), None, 4, None), "v")
    refused(lib.lazyev_append(h, rows(k), rows(k), 0, None), "token count")
    assert lib.lazyev_append(h, rows(k), rows(k), 10 ** 6, None) == binding.ECAPACITY
    assert e.info().n == 0
    with pytest.raises(binding.LazyEvError):
        e.attend(torch.zeros(1, 2, 8, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, 8, D, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        e.append(k, k[:, :, :3])
    with pytest.raises(ValueError):
        e.append(k.transpose(3, 4), k)
    with pytest.raises(ValueError):
        e.append(k, k, positions=torch.zeros(2, 4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        e.norm_rope(x.cpu(), None, x, None)
    with pytest.raises(ValueError):
        e.set_head_norm(torch.zeros(2, D, device="cuda"), None, 1e-6)
    e.append(k, k)
    out = torch.zeros(1, 2, 8, D, dtype=torch.bfloat16, device="cuda")
    assert lib.lazyev_decode_step_rows(h, rows(x[:, :, :1]), rows(k[:, :, :1]), rows(k[:, :, :1]), None, None) == binding.EINVAL
    e.decode_step_rows(x[:, :, 0], k[:, :, 0], k[:, :, 0], out)
    assert e.info().n == 5 and e.info().next_position == 5


# ---- append ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layers,batch,hq,hkv,chunks,dtype,pairs,interleaved,norm", [
    (1, 1, 8, 2, [1], torch.bfloat16, 64, False, True),
    (2, 3, 7, 1, [63, 1, 1, 64, 130], torch.bfloat16, 64, False, True),
    (1, 2, 9, 3, [65, 200], torch.float16, 24, True, True),
    (3, 1, 6, 6, [5, 59, 3], torch.float32, 32, False, False),
    (1, 4, 40, 8, [300], torch.float32, 0, False, False),
])
def test_append_in_chunks(layers, batch, hq, hkv, chunks, dtype, pairs, interleaved, norm):
    g = gen(len(chunks) * 100 + hkv)
    total = sum(chunks)
    e = engine(layers, hq, hkv, batch, total)
    table = np.random.RandomState(3).permutation(e.info().units * e.info().pages_per_unit)
    e.set_page_table(table)
    before = e.state_views()["pages"].clone()
    f = freqs(pairs)
    e.set_rope(f, interleaved=interleaved)
    qkv = randn(g, layers, batch, total, hq + 2 * hkv, D).to(dtype)
    k, v = qkv[..., hq:hq + hkv, :], qkv[..., hq + hkv:, :]
    kw = None
    if norm:
        kw = torch.rand(layers, D, generator=g, device="cuda") + 0.5
        e.set_head_norm(None, kw, 1e-6)
    at = 0
    for c in chunks:
        e.append(k[:, :, at:at + c], v[:, :, at:at + c])
        at += c
        assert e.info().n == e.info().next_position == at
    d = e.dump_state(kv=True)
    units = layers * batch * hkv
    assert np.array_equal(d["pos"], np.tile(np.arange(total), (units, 1)))
    assert not d["ts"].any() and not d["mri"].any() and not d["pbar"].any()
    gv = orc.bf16_bits_to_f64(d["v"]).reshape(layers, batch, hkv, total, D).transpose(0, 1, 3, 2, 4)
    assert np.array_equal(gv, f64(v.to(torch.bfloat16)))
    gk = orc.bf16_bits_to_f64(d["k"]).reshape(layers, batch, hkv, total, D).transpose(0, 1, 3, 2, 4)
    ref, size = rows_ref(k, kw, 1e-6, [np.arange(total)] * batch, f, interleaved)
    assert_rows(torch.from_numpy(gk.copy()), ref, size, torch.bfloat16)
    # nothing outside the appended slots has changed
    pages, ppu = e.state_views()["pages"], e.info().pages_per_unit
    used = torch.zeros(pages.shape[0], 64, dtype=torch.bool, device="cuda")
    for u in range(units):
        for i in range(total):
            used[int(table[u * ppu + i // 64]), i % 64] = True
    keep = ~used[:, None, :, None].expand_as(pages)
    assert torch.equal(pages[keep], before[keep])


def test_append_equals_prefill_and_continues_a_decoded_cache():
    """Rows that need no work: append is prefill bit for bit.  After decode steps it takes TS = t and the next positions."""
    g = gen(8)
    L, B, Hq, Hkv, n = 2, 2, 8, 2, 150
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    a, b = engine(L, Hq, Hkv, B, 400), engine(L, Hq, Hkv, B, 400)
    a.prefill(k, v)
    b.append(k.transpose(2, 3)[:, :, :100], v.transpose(2, 3)[:, :, :100])
    b.append(k.transpose(2, 3)[:, :, 100:], v.transpose(2, 3)[:, :, 100:])
    o1, o2 = (torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for step in range(3):
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        a.decode_step(q, kn, vn, o1)
        b.decode_step_rows(q, kn, vn, o2)
        assert torch.equal(o1, o2)
    x, y = a.dump_state(kv=True), b.dump_state(kv=True)
    for name in ("pos", "ts", "mri", "pbar", "k", "v"):
        assert np.array_equal(x[name], y[name]), name
    b.append(k.transpose(2, 3)[:, :, :5], v.transpose(2, 3)[:, :, :5])
    d = b.dump_state()
    assert np.array_equal(d["pos"][0], np.arange(n + 8)) and np.all(d["ts"][:, -5:] == 3) and not d["mri"][:, -5:].any()
    b.decode_step(q, kn, vn, o2)
    d = b.dump_state()
    assert d["pos"][0, -1] == n + 8 and d["ts"][0, -1] == 4 and b.info().next_position == n + 9


# ---- attention over a shared prefix -----------------------------------------------------------------------------------

def attend_ref(q, kp, vp, ko, vo):
    """out [L, B, Hq, D], sum p |v| of the same shape, pbar [L, B, Hkv, n]; q [L, B, Hq, D], k / v [L, P, Hkv, N, D] and [L, B, Hkv, n, D]."""
    L, B, Hq, _ = q.shape
    P, Hkv = kp.shape[1:3]
    R, G, N = B // P, Hq // Hkv, kp.shape[3]
    q, kp, vp, ko, vo = (x.double() for x in (q, kp, vp, ko, vo))
    k = torch.cat((kp.repeat_interleave(R, 1), ko), 3)
    v = torch.cat((vp.repeat_interleave(R, 1), vo), 3)
    s = (q.view(L, B, Hkv, G, D) @ k.transpose(-1, -2)) / math.sqrt(D)
    p = torch.softmax(s, -1)
    return (p @ v).view(L, B, Hq, D), (p @ v.abs()).view(L, B, Hq, D), p[..., N:].mean(3)


def assert_attend(out, pbar, ref, size, ref_pbar):
    err = (out.double() - ref).abs()
    tol = 2.0 ** -8 * ref.abs() + 2.0 ** -13 * size + 1e-30
    assert bool((err <= tol).all()), f"worst {float((err / tol).max())} of the tolerance"
    if ref_pbar.numel():
        r = ref_pbar.reshape(pbar.shape)
        err = (pbar.double() - r).abs()
        assert bool((err <= 2.0 ** -13 * r + 1e-30).all()), f"pbar: worst {float((err / (2.0 ** -13 * r + 1e-30)).max())}"


def prefixed(g, L, B, P, Hq, Hkv, N, n, kp=None, vp=None, ko=None, vo=None, tables=True):
    kp = randn(g, L, P, Hkv, N, D) if kp is None else kp
    vp = randn(g, L, P, Hkv, N, D) if vp is None else vp
    ko = randn(g, L, B, Hkv, n, D) if ko is None else ko
    vo = randn(g, L, B, Hkv, n, D) if vo is None else vo
    pre, own = engine(L, Hq, Hkv, P, N), engine(L, Hq, Hkv, B, n)
    if tables:
        for e in (pre, own):
            e.set_page_table(np.random.RandomState(N + n).permutation(e.info().units * e.info().pages_per_unit))
    pre.prefill(kp, vp)
    own.attach_prefix(pre)
    if n:
        own.prefill(ko, vo)
    return pre, own, kp, vp, ko, vo


def check_attend(own, q, kp, vp, ko, vo):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    own.attend(q, out)
    own.synchronize()
    assert_attend(out, own.state_views()["pbar"][:, :own.info().n], *attend_ref(q, kp, vp, ko, vo))
    return out


@pytest.mark.parametrize("L,B,P,Hq,Hkv,N,n", [
    (1, 1, 1, 1, 1, 1, 0),              # one key in all
    (1, 4, 1, 8, 2, 1, 1),
    (1, 4, 2, 8, 2, 63, 1),
    (2, 6, 3, 6, 6, 64, 65),            # one query head per KV head
    (1, 3, 1, 9, 3, 127, 0),
    (1, 40, 1, 8, 1, 128, 5),           # three row tiles: a pair and a single one
    (1, 36, 1, 7, 1, 129, 64),          # two row tiles with unused rows, a tile of one key
    (1, 37, 1, 5, 1, 1000, 3),
    (2, 64, 2, 16, 2, 4100, 130),       # several blocks per item, two streams per block
    (1, 2, 1, 28, 4, 20001, 70),        # many blocks per item
    (3, 48, 3, 40, 8, 777, 200),
    (1, 150, 1, 2, 2, 300, 20),
    (28, 32, 2, 28, 4, 300, 10),        # more items than blocks
    (5, 1, 1, 12, 2, 200, 700),         # own tokens longer than the prefix, no sharing
    (1, 260, 1, 4, 4, 513, 0),
    (4, 40, 1, 8, 4, 200, 0),           # many units with short own caches: a warp each
    (6, 40, 2, 16, 2, 200, 1),
    (4, 40, 1, 28, 4, 1000, 16),
    (4, 150, 1, 5, 1, 5000, 17),        # many partial sums per row
    (16, 40, 1, 12, 2, 70, 65),
    (16, 40, 1, 7, 7, 70, 240),
    (16, 40, 1, 6, 2, 70, 255),
    (30, 45, 1, 40, 8, 70, 383),        # several units per warp
    (30, 45, 1, 3, 1, 70, 384),
    (30, 45, 3, 9, 3, 70, 385),         # one token too long for it
    (1, 56, 1, 32, 8, 64, 128),         # three units per SM: a warp each up to here,
    (1, 56, 1, 32, 8, 64, 129),         # a block each from here
    (1, 73, 1, 32, 8, 64, 129),         # just below and at four units per SM
    (1, 74, 1, 32, 8, 64, 129),
])
def test_attend_against_64_bits(L, B, P, Hq, Hkv, N, n):
    g = gen(N * 7 + n)
    pre, own, *kv = prefixed(g, L, B, P, Hq, Hkv, N, n)
    assert own.info().prefix_tokens == N and own.info().next_position == N + n
    q = randn(g, L, B, Hq, D)
    a = check_attend(own, q, *kv)
    check_attend(own, 3 * randn(g, L, B, Hq, D), *kv)          # sharper rows
    b = check_attend(own, q, *kv)
    assert torch.equal(a, b)                                   # the same bits in every run
    assert own.info().n == n and own.info().t == 0


@pytest.mark.parametrize("rows", ["pair", "single"])
@pytest.mark.parametrize("order", ["rising", "falling", "late"])
def test_references_that_have_to_rise(rows, order):
    """Logits that climb over hundreds of log2 units along the prefix: the running reference is raised tile after tile
    and O rescaled; or only a key at the very end matters; or the first one decides all."""
    g = gen(3)
    B, G, N, n = (40, 8, 2000, 40) if rows == "pair" else (6, 8, 2000, 40)
    u = torch.randn(D, generator=g, device="cuda")
    u = u / u.norm()
    slope = torch.linspace(-200, 200, N, device="cuda")
    slope = {"rising": slope, "falling": slope.flip(0), "late": torch.where(torch.arange(N, device="cuda") == N - 1, 300.0, 0.0)}[order]
    kp = (0.3 * torch.randn(1, 1, 1, N, D, generator=g, device="cuda") + slope[:, None] * u).to(torch.bfloat16)
    q = ((1 + torch.rand(1, B, G, 1, generator=g, device="cuda")) * 4 * u + 0.1 * torch.randn(1, B, G, D, generator=g, device="cuda")).to(torch.bfloat16)
    pre, own, *kv = prefixed(g, 1, B, 1, G, 1, N, n, kp=kp)
    check = attend_ref(q, *kv)
    out = torch.empty_like(q)
    own.attend(q, out)
    own.synchronize()
    # logits of up to 800: 128 * 2^-23 of them would be 2^-7; the products of a large logit nearly all have one sign and their
    # sum is off by about 2^-22 of it, hence exp by 2^-12 at 800, and the two sides of the softmax by 2^-11
    err = (out.double() - check[0]).abs()
    assert bool((err <= 2.0 ** -8 * check[0].abs() + 2.0 ** -10 * check[1]).all())
    total = own.state_views()["pbar"][:, :n].double().sum(-1)
    assert bool(((total - check[2].reshape(total.shape[0], n).sum(-1)).abs() <= 2.0 ** -10).all())


def test_prefix_tail_and_padding_hold_no_poison():
    """Slots behind the prefix's last token may hold anything from an earlier sequence, NaN and infinities included."""
    g = gen(4)
    L, B, Hq, Hkv, N, n = 1, 5, 8, 2, 70, 3
    pre, own = engine(L, Hq, Hkv, 1, 128), engine(L, Hq, Hkv, B, n)
    bad = torch.full((L, 1, Hkv, 128, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    bad[..., 100:, :] = float("inf")
    pre.prefill(bad, bad)
    pre.reset()
    kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
    pre.append(kp.transpose(2, 3), vp.transpose(2, 3))
    own.attach_prefix(pre)
    ko, vo = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    own.prefill(ko, vo)
    check_attend(own, randn(g, L, B, Hq, D), kp, vp, ko, vo)
    # a key that is infinite in one head poisons that head's rows only
    kp[0, 0, 1, 5] = float("inf")
    own.reset()
    pre.reset()
    pre.prefill(kp, vp)
    own.attach_prefix(pre)
    q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    own.attend(q, out)
    own.synchronize()
    ref, size, _ = attend_ref(q, kp, vp, ko[..., :0, :], vo[..., :0, :])
    assert not bool(torch.isfinite(out[:, :, 4:]).any()) and bool(torch.isnan(ref[:, :, 4:]).all())
    err = (out[:, :, :4].double() - ref[:, :, :4]).abs()
    assert bool((err <= 2.0 ** -8 * ref[:, :, :4].abs() + 2.0 ** -13 * size[:, :, :4]).all())


def test_prefix_equals_one_cache_within_rounding_and_detach_ends_it():
    """The same tokens as prefix + own cache and as one cache: outputs agree to the tolerance, and so do probabilities."""
    g = gen(6)
    L, B, Hq, Hkv, N, n = 2, 4, 28, 4, 500, 90
    pre, own, kp, vp, ko, vo = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    whole = engine(L, Hq, Hkv, B, N + n)
    whole.prefill(torch.cat((kp.expand(L, B, Hkv, N, D), ko), 3).contiguous(), torch.cat((vp.expand(L, B, Hkv, N, D), vo), 3).contiguous())
    q, a, b = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    own.attend(q, a)
    whole.attend(q, b)
    own.synchronize(), whole.synchronize()
    ref, size, pb = attend_ref(q, kp, vp, ko, vo)
    assert_attend(a, own.state_views()["pbar"][:, :n], ref, size, pb)
    assert_attend(b, whole.state_views()["pbar"][:, N:N + n], ref, size, pb)
    own.detach_prefix()
    own.detach_prefix()                                        # nothing left to detach
    own.attend(q, a)
    own.synchronize()
    none = kp[:, :, :, :0].expand(L, B, Hkv, 0, D)
    assert_attend(a, own.state_views()["pbar"][:, :n], *attend_ref(q, none, none, ko, vo))
    assert own.info().prefix_tokens == 0 and own.info().next_position == N + n


def test_sharing_rules():
    g = gen(2)
    pre, own, *_ = prefixed(g, 1, 4, 2, 8, 2, 30, 5)
    lib, E = binding.lib(), binding
    q, kn, o4 = randn(g, 1, 2, 8, D), randn(g, 1, 2, 2, D), torch.empty(1, 4, 8, D, dtype=torch.bfloat16, device="cuda")
    o2 = torch.empty(1, 2, 8, D, dtype=torch.bfloat16, device="cuda")

    def code(f, *a):
        with pytest.raises(E.LazyEvError) as err:
            f(*a)
        return err.value.code

    # the prefix may be read but not changed
    pre.attend(q, o2)
    assert code(pre.decode_step, q, kn, kn, o2) == E.ESTATE
    assert code(pre.decode_step_rows, q, kn, kn, o2) == E.ESTATE
    assert code(pre.append, kn.unsqueeze(2), kn.unsqueeze(2)) == E.ESTATE
    assert code(pre.evict) == E.ESTATE and code(pre.evict_static) == E.ESTATE
    assert code(pre.reset) == E.ESTATE and code(pre.close) == E.ESTATE
    assert pre.info().n == 30
    # what does not fit
    assert code(own.attach_prefix, pre) == E.ESTATE            # one is attached
    three = engine(1, 8, 2, 3, 5)
    assert code(three.attach_prefix, pre) == E.EINVAL          # 3 sequences, 2 prefixes
    assert code(engine(1, 16, 2, 4, 5).attach_prefix, pre) == E.EINVAL
    assert code(engine(2, 8, 2, 4, 5).attach_prefix, pre) == E.EINVAL
    empty, other = engine(1, 8, 2, 2, 5), engine(1, 8, 2, 4, 5)
    assert code(other.attach_prefix, empty) == E.ESTATE        # nothing in it
    assert code(other.attach_prefix, own) == E.ESTATE          # has a prefix itself
    empty.append(kn.unsqueeze(2), kn.unsqueeze(2))
    assert code(pre.attach_prefix, empty) == E.ESTATE          # is one itself
    assert lib.lazyev_attach_prefix(other._h, pre._h, 8) == E.EINVAL       # misaligned workspace
    assert lib.lazyev_attach_prefix(other._h, None, None) == E.EINVAL
    assert lib.lazyev_attach_prefix(pre._h, pre._h, 256) == E.EINVAL
    assert code(own.prefill_observed, q, kn, kn, o2) == E.ESTATE
    q_odd = torch.empty(4 * 8 * D + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 8, D)
    assert code(own.attend, q_odd, o4) == E.EINVAL             # the prefix launch wants 16 bytes
    copy = engine(1, 8, 2, 4, 5)
    assert code(copy.copy_state_from, own) == E.ESTATE
    copy.attach_prefix(pre)
    copy.copy_state_from(own)
    # the last user lets go
    q4 = randn(g, 1, 4, 8, D)
    o5 = torch.empty_like(o4)
    own.attend(q4, o4)
    copy.attend(q4, o5)
    torch.cuda.synchronize()
    assert torch.equal(o4, o5)
    own.reset()
    assert code(pre.reset) == E.ESTATE
    copy.close()
    pre.reset()
    assert own.info().prefix_tokens == 0


def test_step_entry_points_agree_with_a_prefix():
    """decode_step, its host-buffer forms, decode_step_rows and both append routes: one result, bit for bit."""
    g = gen(11)
    L, B, Hq, Hkv, N, n = 2, 6, 28, 4, 333, 70
    kp, vp = randn(g, L, 2, Hkv, N, D), randn(g, L, 2, Hkv, N, D)
    ko, vo = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    pre = engine(L, Hq, Hkv, 2, N)
    pre.prefill(kp, vp)
    engines = {}
    for name in ("device", "separate", "rows", "host", "async"):
        e = binding.Engine(L, Hq, Hkv, D, 80, 16, 1e-3, batch=B)
        e.attach_prefix(pre)
        e.prefill(ko, vo)
        engines[name] = e
    engines["separate"].set_fused_append(False)
    outs = {k: torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda") for k in ("device", "separate", "rows")}
    for step in range(20):                                     # an eviction at step 16
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        engines["device"].decode_step(q, kn, vn, outs["device"])
        engines["separate"].decode_step(q, kn, vn, outs["separate"])
        engines["rows"].decode_step_rows(q, kn, vn, outs["rows"])
        host = [x.cpu().pin_memory() for x in (q, kn, vn)]
        ho, ha = torch.empty(L, B, Hq, D, dtype=torch.bfloat16).pin_memory(), torch.empty(L, B, Hq, D, dtype=torch.bfloat16).pin_memory()
        engines["host"].decode_step_host(*(x for x in host), ho)
        engines["async"].decode_step_host_async(*(x for x in host), ha)
        engines["async"].host_wait(0)
        torch.cuda.synchronize()
        for name, x in (("separate", outs["separate"]), ("rows", outs["rows"]), ("host", ho), ("async", ha)):
            assert torch.equal(outs["device"].cpu(), x.cpu()), (name, step)
    want = engines["device"].dump_state(kv=True)
    assert want["n"] < n + 20 and engines["device"].info().evictions == 1
    for name, e in engines.items():
        got = e.dump_state(kv=True)
        for f in ("pos", "ts", "mri", "pbar", "k", "v"):
            assert np.array_equal(want[f], got[f]), (name, f)


@pytest.mark.parametrize("n,ranges", [(64, 1), (400, 3)])       # short own caches are one launch, longer ones a walk of 13 rounds
def test_wide_host_step_with_a_prefix(n, ranges):
    """More units than blocks: the host-buffer step runs in unit ranges, the prefix launch once for all of them."""
    g = gen(12)
    L, B, Hq, Hkv, N = 14, 32, 28, 4, 200
    pre, own, *kv = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    twin = engine(L, Hq, Hkv, B, n)
    twin.attach_prefix(pre)
    twin.prefill(kv[2], kv[3])
    q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
    out = torch.empty_like(q)
    ho = torch.empty(q.shape, dtype=torch.bfloat16).pin_memory()
    own.decode_step_host(*(x.cpu().pin_memory() for x in (q, kn, vn)), ho)
    twin.decode_step(q, kn, vn, out)
    twin.synchronize()
    assert own.info().host_ranges >= ranges and torch.equal(out.cpu(), ho)
    ref = attend_ref(q, kv[0], kv[1], torch.cat((kv[2], kn.unsqueeze(3)), 3), torch.cat((kv[3], vn.unsqueeze(3)), 3))
    own_pb = own.state_views()["pbar"][:, :n + 1]
    twin_pb = twin.state_views()["pbar"][:, :n + 1]
    assert_attend(out, twin_pb, *ref)
    assert torch.equal(own_pb, twin_pb)


@pytest.mark.parametrize("splits", [1, 2, 5])
def test_prefix_with_forced_clusters(splits):
    g = gen(13)
    pre, own, *kv = prefixed(g, 1, 3, 1, 8, 2, 2500, 700)
    own.set_splits(splits)
    check_attend(own, randn(g, 1, 3, 8, D), *kv)
    assert own.info().splits == splits


def test_two_users_on_streams_of_their_own():
    g = gen(14)
    L, Hq, Hkv, N = 1, 32, 8, 3000
    kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
    s0, s1, s2 = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    pre = engine(L, Hq, Hkv, 1, N, stream=s0)
    pre.prefill(kp, vp)
    users = [engine(L, Hq, Hkv, 8, 50, stream=s) for s in (s1, s2)]
    data = [(randn(g, L, 8, Hq, D), randn(g, L, 8, Hkv, 50, D), randn(g, L, 8, Hkv, 50, D)) for _ in users]
    outs = [torch.empty(L, 8, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in users]
    torch.cuda.synchronize()
    for e, (q, k, v) in zip(users, data):
        e.attach_prefix(pre)
        e.prefill(k, v)
    for _ in range(5):
        for e, (q, _, _), o in zip(users, data, outs):
            e.attend(q, o)
    for e, (q, k, v), o in zip(users, data, outs):
        e.synchronize()
        assert_attend(o, e.state_views()["pbar"][:, :50], *attend_ref(q, kp, vp, k, v))
    # the prefix changes only after its readers are done: reset and reload right behind their queued work
    for e, (q, _, _), o in zip(users, data, outs):
        for _ in range(20):
            e.attend(q, o)
        e.detach_prefix()
    pre.reset()
    pre.prefill(torch.zeros_like(kp), torch.zeros_like(vp))
    torch.cuda.synchronize()
    for (q, k, v), o in zip(data, outs):
        ref, size, _ = attend_ref(q, kp, vp, k, v)
        assert bool(((o.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -13 * size).all())


def test_captured_and_replayed():
    """norm_rope and attend in a CUDA graph: new queries in the same buffers, replayed."""
    g = gen(15)
    L, B, Hq, Hkv, N, n = 1, 6, 8, 2, 400, 20
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        pre, own, *kv = prefixed(g, L, B, 1, Hq, Hkv, N, n)
        own.set_rope(freqs(64))
        raw, q, out = randn(g, L, B, 1, Hq, D), torch.empty(L, B, 1, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
        pos = torch.full((B, 1), N + n - 1, dtype=torch.int32, device="cuda")

        def step():
            own.norm_rope(raw, None, q, None, positions=pos)
            own.attend(q, out)

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in (1, 2):
            raw.copy_(randn(gen(seed), L, B, 1, Hq, D))
            pos.fill_(seed * 1000)
            graph.replay()
            stream.synchronize()
            got_q, got = q.clone(), out.clone()
            ref, size = rows_ref(raw, None, 0, [[seed * 1000]] * B, freqs(64))
            assert_rows(got_q, ref, size, torch.bfloat16)
            assert_attend(got, own.state_views()["pbar"][:, :n], *attend_ref(got_q[:, :, 0], *kv))


@pytest.mark.parametrize("L,N,limits", [(1, 4000, (0,)), (1, 60000, (1, 3)),     # blocks have one key tile each / six and more
                                        (16, 300, (1,))])                         # a warp per unit in the decode launch
def test_a_prefix_launch_that_starves_reports_and_recovers(L, N, limits):
    """The producer of the prefix kernel stops after some key tiles: bounded waits run out, the status word tells, and
    after a reset the handle works again."""
    g = gen(16)
    pre, own, *kv = prefixed(g, L, 40, 1, 8, 1, N, 100)
    q = randn(g, L, 40, 8, D)
    out = torch.empty_like(q)
    own.set_wait_limit(0.002)
    for tiles in limits:
        own.debug_starve_page_ring(tiles)
        own.attend(q, out)
        with pytest.raises(binding.LazyEvError) as err:
            own.synchronize()
        assert err.value.code == binding.EDEVICE
        own.debug_starve_page_ring(-1)
        own.reset()
        own.attach_prefix(pre)
        own.prefill(kv[2], kv[3])
    own.set_wait_limit(2.0)
    check_attend(own, q, *kv)


def test_prefix_pages_behind_four_gigabytes():
    g = gen(21)
    L, B, Hq, Hkv, N, n = 1, 3, 8, 4, 500, 10
    pre = binding.Engine(L, Hq, Hkv, D, 2 ** 22, 64, 2.0, batch=1)        # 65 537 pages per unit
    own = engine(L, Hq, Hkv, B, n)
    inf = pre.info()
    assert inf.units * inf.pages_per_unit * 32768 > 2 ** 32
    pre.set_page_table(np.arange(inf.units * inf.pages_per_unit)[::-1].copy())
    kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
    ko, vo = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    pre.prefill(kp, vp)
    own.attach_prefix(pre)
    own.prefill(ko, vo)
    check_attend(own, randn(g, L, B, Hq, D), kp, vp, ko, vo)


def test_stale_slots_of_the_own_cache_hold_no_poison():
    """NaN and infinite rows of an earlier sequence in the slots behind the last token: append, attend, decode and the prompt's
    replay see nothing of them, with and without a prefix."""
    g = gen(22)
    L, B, Hq, Hkv, N = 1, 5, 8, 2, 100
    kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
    pre = engine(L, Hq, Hkv, 1, N)
    pre.prefill(kp, vp)
    none = kp[:, :, :, :0].expand(L, B, Hkv, 0, D)
    for shared in (False, True):
        e = engine(L, Hq, Hkv, B, 200)
        bad = torch.full((L, B, Hkv, 200, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        bad[..., 64:, :] = float("-inf")
        e.prefill(bad, bad)
        for n in (1, 7, 16, 63, 64, 65, 130):
            e.reset()
            if shared:
                e.attach_prefix(pre)
            k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
            e.append(k.transpose(2, 3), v.transpose(2, 3))
            q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
            pk, pv = (kp, vp) if shared else (none, none)
            check_attend(e, q, pk, pv, k, v)
            kn, vn = randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
            e.decode_step(q, kn, vn, out)
            e.synchronize()
            ref = attend_ref(q, pk, pv, torch.cat((k, kn.unsqueeze(3)), 3), torch.cat((v, vn.unsqueeze(3)), 3))
            assert_attend(out, e.state_views()["pbar"][:, :n + 1], *ref)


def test_decoding_starts_with_no_own_token():
    g = gen(23)
    L, B, Hq, Hkv, N = 2, 6, 14, 2, 129
    pre, own, kp, vp, ko, vo = prefixed(g, L, B, 2, Hq, Hkv, N, 0)
    ks, vs = [], []
    for step in range(3):
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        ks.append(kn), vs.append(vn)
        out = torch.empty_like(q)
        if step < 2:
            own.decode_step(q, kn, vn, out)
        else:
            own.decode_step_rows(q, kn, vn, out)
        own.synchronize()
        assert_attend(out, own.state_views()["pbar"][:, :step + 1], *attend_ref(q, kp, vp, torch.stack(ks, 3), torch.stack(vs, 3)))
        if step == 0:
            with pytest.raises(binding.LazyEvError):
                own.prefill(ko, vo)                            # it holds tokens now
    d = own.dump_state()
    assert np.array_equal(d["pos"][0], N + np.arange(3)) and np.array_equal(d["ts"][0], [1, 2, 3])


def test_resume_behind_a_prefix():
    """A snapshot of sequences that began with no prompt of their own goes into another handle behind the same prefix."""
    g = gen(24)
    L, B, Hq, Hkv, N = 1, 4, 8, 2, 90
    pre, a, *_ = prefixed(g, L, B, 1, Hq, Hkv, N, 0)
    out = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    for _ in range(5):
        a.decode_step(randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D), out)
    snap = a.dump_state(kv=True)
    b = engine(L, Hq, Hkv, B, 5)
    with pytest.raises(binding.LazyEvError):
        b.load_state(snap, 0)                                  # without a prefix there has to be a prompt
    b.attach_prefix(pre)
    b.load_state(snap, 0)
    assert b.info().next_position == a.info().next_position == N + 5
    q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
    out2 = torch.empty_like(out)
    a.decode_step(q, kn, vn, out)
    b.decode_step(q, kn, vn, out2)
    x, y = a.dump_state(kv=True), b.dump_state(kv=True)
    assert torch.equal(out, out2)
    for name in ("pos", "ts", "mri", "pbar", "k", "v"):
        assert np.array_equal(x[name], y[name]), name


def test_rows_of_extreme_size():
    """Zero rows, rows near the largest and smallest bf16, and a row with an infinity: the norm's factor meets the elements first,
    as in the formula in 32 bits, and rows do not touch each other."""
    e = engine(1, 4, 4, 1, 1)
    e.set_rope(freqs(64))
    w = torch.full((1, D), 1.5, device="cuda")
    e.set_head_norm(w, None, 1e-6)
    x = torch.ones(1, 1, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    x[..., 0, :], x[..., 1, :], x[..., 2, :] = 0.0, 1e18, 1e-30
    x[..., 3, 7] = float("inf")
    out = torch.empty_like(x)
    e.norm_rope(x, None, out, None, first_position=3)
    e.synchronize()
    finite = x[..., :3, :]
    ref, size = rows_ref(finite, w, 1e-6, [[3]], freqs(64))
    assert_rows(out[..., :3, :], ref, size, torch.bfloat16)
    assert not bool(torch.isfinite(out[..., 3, 7]).any())


def test_range_checked_build():
    """The same tests through the build whose kernels check every slot, page and work index."""
    import os
    import subprocess
    import sys
    if binding.debug_bounds_requested():
        pytest.skip("already inside the range-checked run")
    res = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-m", "gpu", "-k",
                          "64_bits or chunks or many_tokens or rise or poison or serving or clusters or entry_points"],
                         env=dict(os.environ, LAZYEV_DEBUG_BOUNDS="1"), capture_output=True, text=True,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-2000:]
    assert " passed" in res.stdout and "failed" not in res.stdout


# ---- together ------------------------------------------------------------------------------------------------------------

def test_serving_run_from_projections_to_evictions():
    """Two prompts, three samples of each: the prompts' projected rows are appended in chunks, the samples attach, load a
    few tokens of their own and decode from projected rows across evictions; the last prompt queries are asked again with
    attend.  Every step is held to the 64-bit oracle, whose bookkeeping takes the GPU's probabilities."""
    g = gen(17)
    L, P, R, Hq, Hkv, N, W, budget = 2, 2, 3, 14, 2, 201, 16, 48
    B, G = P * R, Hq // Hkv
    alpha, eps = 4e-3, 1e-6
    f = freqs(64, 5e5)
    qw, kw = (torch.rand(L, D, generator=g, device="cuda") + 0.5 for _ in range(2))
    pre = engine(L, Hq, Hkv, P, N)
    own = binding.Engine(L, Hq, Hkv, D, budget, W, alpha, batch=B)
    for e in (pre, own):
        e.set_rope(f)
        e.set_head_norm(qw, kw, eps)
    qkv = randn(g, L, P, N, Hq + 2 * Hkv, D)
    for a, b in ((0, 100), (100, 101), (101, N)):
        pre.append(qkv[:, :, a:b, Hq:Hq + Hkv], qkv[:, :, a:b, Hq + Hkv:])
    d = pre.dump_state(kv=True)
    kp, vp = orc.bf16_bits_to_f64(d["k"]), orc.bf16_bits_to_f64(d["v"])
    ref, size = rows_ref(qkv[..., Hq:Hq + Hkv, :], kw, eps, [np.arange(N)] * P, f)
    assert_rows(torch.from_numpy(kp.reshape(L, P, Hkv, N, D).transpose(0, 1, 3, 2, 4).copy()), ref, size, torch.bfloat16)
    own.attach_prefix(pre)
    units = [orc.PrefixedUnit(kp[((u // Hkv // B) * P + u // Hkv % B // R) * Hkv + u % Hkv], vp[((u // Hkv // B) * P + u // Hkv % B // R) * Hkv + u % Hkv],
                              N, G, D, budget, W, alpha) for u in range(L * B * Hkv)]

    def hold(out, ref_out, pbar, ref_pbar):
        assert np.all(np.abs(out - ref_out) <= 2e-3 + 1e-2 * np.abs(ref_out))
        assert np.all(np.abs(pbar - ref_pbar) <= 1e-6 + 2.0 ** -13 * ref_pbar)

    # the queries of the prompts' last token, over the prompt alone
    q1 = torch.empty(L, P, 1, Hq, D, dtype=torch.bfloat16, device="cuda")
    pre.norm_rope(qkv[:, :, N - 1:, :Hq], None, q1, None, first_position=N - 1)
    qb, out = q1[:, :, 0].repeat_interleave(R, 1).contiguous(), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    own.attend(qb, out)
    own.synchronize()
    qh, oh = f64(qb).reshape(-1, G, D), f64(out).reshape(-1, G, D)
    for u, unit in enumerate(units):
        hold(oh[u], unit.look(qh[u])[0], np.zeros(0), np.zeros(0))

    extra = randn(g, L, B, 5, Hq + 2 * Hkv, D)
    own.append(extra[..., Hq:Hq + Hkv, :], extra[..., Hq + Hkv:, :])
    d = own.dump_state(kv=True)
    for u, unit in enumerate(units):
        unit.load(orc.bf16_bits_to_f64(d["k"][u]), orc.bf16_bits_to_f64(d["v"][u]))
        assert np.array_equal(unit.pos, d["pos"][u])
    for step in range(1, 7 * W + 3):
        x = randn(g, L, B, Hq + 2 * Hkv, D)
        before = own.info()
        assert before.next_position == N + 5 + step - 1
        at = [[before.next_position]] * B
        own.decode_step_rows(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], out)
        evicted = own.info().n < before.n + 1
        d = own.dump_state(kv=True)
        # the oracle sees the rows as the cache holds them; what it holds is checked against the formula
        rq, sq = rows_ref(x[:, :, None, :Hq], qw, eps, at, f)
        rk, sk = rows_ref(x[:, :, None, Hq:Hq + Hkv], kw, eps, at, f)
        rv = f64(x[:, :, Hq + Hkv:]).reshape(-1, D)
        assert_rows(torch.from_numpy(orc.bf16_bits_to_f64(d["k"][:, -1])), rk.reshape(-1, D), sk.reshape(-1, D), torch.bfloat16)
        assert np.array_equal(orc.bf16_bits_to_f64(d["v"][:, -1]), rv)
        qo = torch.empty(L, B, 1, Hq, D, dtype=torch.bfloat16, device="cuda")
        own.norm_rope(x[:, :, None, :Hq], None, qo, None, first_position=before.next_position)
        own.synchronize()
        qh, oh = f64(qo).reshape(-1, G, D), f64(out).reshape(-1, G, D)
        for u, unit in enumerate(units):
            o, pb = unit.attend(qh[u], orc.bf16_bits_to_f64(d["k"][u, -1]), rv[u])
            if not evicted:
                hold(oh[u], o, d["pbar"][u], pb)
                unit.track(d["pbar"][u])
            else:
                hold(oh[u], o, np.zeros(0), np.zeros(0))
                unit.track(pb)                                  # (its probabilities moved with the eviction)
            assert unit.evict_due() == evicted
            if evicted:
                unit.evict_if_due()
                gap = set(unit.pos) ^ set(d["pos"][u])
                assert len(gap) <= 2, gap                       # a probability within rounding of alpha may flip one token
                if gap:
                    pytest.fail(f"evict sets differ: {gap}")
            assert np.array_equal(unit.pos, d["pos"][u]) and np.array_equal(unit.TS, d["ts"][u]) and np.array_equal(unit.MRI, d["mri"][u])
    assert own.info().evictions >= 4 and own.info().n <= budget + W
