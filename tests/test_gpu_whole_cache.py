"""The operators on a whole cache against plain 64-bit forms: attention of a chunk of tokens, the weights that tokens
receive, eviction by them and into another cache, attention over selected blocks; and a run of them together.

Tolerances.  A rounding to a type is off by at most eps / 2 of the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).  Besides it:
* logits: as for a decode step, 2^-13 of sum_i p_i |v_i| for an output, 2^-13 of a probability.
* a chunk's value product takes its weights in bf16, each off by at most 2^-8 of itself: 2^-8 of sum_i p_i |v_i| for an output.  The
  two and the output's own rounding multiply: 2^-8 of either bounds the product of two of them.
* a token's weight is a sum of positive probabilities, 32 at a time and then tile by tile: below 2^-14 beside the probabilities' 2^-13.
* selections, positions, moved rows and weights are exact.
"""
import math

import numpy as np
import pytest
import torch

from oracle import lazyev_oracle as orc
from paper_2506_15969_b200 import binding
from tests.test_gpu_operators import TYPES, attend_ref, engine, freqs, gen, randn, rows_ref, assert_rows

pytestmark = pytest.mark.gpu

D = 128


# ---- a chunk ----------------------------------------------------------------------------------------------------------

def chunk_ref(q, k, v, T, kp=None, vp=None):
    """out [L, B, T, Hq, D], sum p |v| of the same shape, weights [units, n]; q [L, B, T, Hq, D], k / v [L, B, Hkv, n, D] of all own
    tokens, kp / vp [L, P, Hkv, N, D].  What a row does not see is cut off, not multiplied by zero."""
    L, B, _, Hq, _ = q.shape
    Hkv, n = k.shape[2:4]
    G, N = Hq // Hkv, 0 if kp is None else kp.shape[3]
    out, size = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape, dtype=torch.float64, device="cuda")
    weights = torch.zeros(L, B, Hkv, n, dtype=torch.float64, device="cuda")
    bad = not bool(torch.isfinite(v).all())
    for l in range(L):
        for b in range(B):
            for h in range(Hkv):
                kk, vv = k[l, b, h].double(), v[l, b, h].double()
                if N:
                    p = b // (B // kp.shape[1])
                    kk, vv = torch.cat((kp[l, p, h].double(), kk)), torch.cat((vp[l, p, h].double(), vv))
                x = torch.einsum("tgd,jd->tgj", q[l, b, :, h * G:(h + 1) * G].double(), kk) / math.sqrt(D)
                sees = torch.ones(T, N + n, dtype=torch.bool, device="cuda").tril(N + n - T)
                x = x.masked_fill(~sees[:, None], -math.inf)
                p = torch.softmax(x, -1)
                p = torch.where(sees[:, None], p, 0.0)
                if bad:
                    for t in range(T):
                        to = N + n - T + t + 1
                        out[l, b, t, h * G:(h + 1) * G] = p[t, :, :to] @ vv[:to]
                        size[l, b, t, h * G:(h + 1) * G] = p[t, :, :to] @ vv[:to].abs()
                else:
                    out[l, b, :, h * G:(h + 1) * G] = p @ vv
                    size[l, b, :, h * G:(h + 1) * G] = p @ vv.abs()
                weights[l, b, h] = p[..., N:].sum((0, 1)) / G
    return out, size, weights.view(-1, n)


def assert_chunk(got, ref, size, weights=None, ref_weights=None):
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(ref)), "rows that are finite"
    ok = torch.isfinite(ref)
    tol = (TYPES[assert_chunk.dtype] * ref.abs() + (2.0 ** -8 + 2.0 ** -13) * size) * (1 + 2.0 ** -7) + 1e-30
    worst = float(((got - ref).abs()[ok] / tol[ok]).max()) if bool(ok.any()) else 0.0
    assert worst <= 1, f"worst {worst} of the tolerance"
    if weights is not None:
        tol = (2.0 ** -13 + 2.0 ** -14) * ref_weights + 1e-30
        worst = float(((weights.double() - ref_weights).abs() / tol).max())
        assert worst <= 1, f"weights: worst {worst} of the tolerance"


def run_chunk(e, q, out_dtype=torch.bfloat16, **kw):
    out = torch.full(q.shape, 7.0, dtype=out_dtype, device="cuda")
    e.attend_chunk(q, out, **kw)
    e.synchronize()
    assert_chunk.dtype = out_dtype
    return out


def loaded(g, L, B, Hq, Hkv, n, k=None, v=None, weights=False, **kw):
    e = engine(L, Hq, Hkv, B, n, weights=weights, **kw)
    e.set_page_table(np.random.RandomState(n).permutation(e.info().units * e.info().pages_per_unit))
    k = randn(g, L, B, Hkv, n, D) if k is None else k
    v = randn(g, L, B, Hkv, n, D) if v is None else v
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    return e, k, v


@pytest.mark.parametrize("L,B,Hq,Hkv,context,T,dtype", [
    (1, 1, 1, 1, 0, 1, torch.bfloat16),             # one key in all
    (1, 1, 8, 2, 0, 2, torch.float32),
    (1, 2, 8, 2, 127, 1, torch.bfloat16),           # single tokens around the borders of tiles and pages
    (1, 2, 8, 2, 128, 1, torch.float32),
    (2, 3, 28, 4, 63, 1, torch.float16),
    (1, 1, 5, 1, 20000, 1, torch.bfloat16),         # many blocks per item
    (1, 1, 7, 1, 20001, 3, torch.float32),
    (2, 2, 6, 6, 64, 128, torch.float16),           # one query head per KV head: a whole row tile
    (1, 1, 6, 6, 1, 129, torch.bfloat16),           # a tile and a row
    (1, 3, 9, 3, 0, 300, torch.bfloat16),           # 42 tokens of 3 heads per tile, an odd number of tiles
    (2, 2, 28, 4, 91, 37, torch.float32),           # 18 tokens of 7 heads
    (1, 2, 40, 8, 1000, 51, torch.bfloat16),        # 25 tokens of 5 heads, one behind two tiles
    (1, 4, 16, 2, 33, 65, torch.bfloat16),          # 16 tokens of 8 heads
    (4, 20, 12, 2, 200, 4, torch.bfloat16),         # more items than blocks, one row tile each
    (3, 40, 8, 2, 90, 30, torch.float16),
    (1, 1, 2, 1, 0, 1500, torch.bfloat16),          # a causal triangle, items of 1 to 12 key tiles
    (2, 1, 4, 1, 700, 900, torch.float32),
    (1, 150, 2, 2, 10, 70, torch.bfloat16),
])
@pytest.mark.parametrize("weights", [binding.WEIGHTS_OFF, binding.WEIGHTS_SET])
def test_chunk_against_64_bits(L, B, Hq, Hkv, context, T, dtype, weights):
    g = gen(context * 3 + T)
    e, k, v = loaded(g, L, B, Hq, Hkv, context + T, weights=weights != binding.WEIGHTS_OFF)
    qkv = randn(g, L, B, T, Hq + 3, D)                         # queries as a part of a projection's rows
    q = qkv[..., 1:Hq + 1, :]
    out, size, w = chunk_ref(q, k, v, T)
    before = e.dump_state()
    got = run_chunk(e, q, dtype, weights=weights)
    assert_chunk(got, out, size, *((e.state_views()["weights"][:, :context + T], w) if weights else ()))
    after = e.dump_state()
    assert all(np.array_equal(before[x], after[x]) for x in ("pos", "ts", "mri", "pbar")) and before["n"] == after["n"]
    again = run_chunk(e, q, dtype, weights=weights)
    assert torch.equal(got, again)                             # the same bits every time


@pytest.mark.parametrize("L,B,Hq,Hkv,context,T", [
    (2, 4, 32, 8, 500, 300),                        # two to three items of 5 to 7 key tiles per block, begun and ended inside an item
    (1, 9, 30, 6, 1100, 260),                       # 25 tokens of 5 heads, an odd number of tiles
    (1, 2, 64, 32, 0, 1025),                        # a triangle: items of 1 to 9 key tiles
])
def test_chunk_of_many_items_in_any_order(L, B, Hq, Hkv, context, T):
    """A block works on whole items first, then on the one that it shares with the next block, then on the one before's."""
    g = gen(L + B + Hq + context)
    n = context + T
    e, k, v = loaded(g, L, B, Hq, Hkv, n, weights=True)
    q = randn(g, L, B, T, Hq, D)
    out = run_chunk(e, q, weights=binding.WEIGHTS_SET)
    again = run_chunk(e, q, weights=binding.WEIGHTS_SET)
    assert torch.equal(out, again)
    ref, size, weights = chunk_ref(q, k, v, T)
    assert_chunk(out, ref, size, e.state_views()["weights"][:, :n], weights)


@pytest.mark.parametrize("L,B,Hq,Hkv,context,T,dtype", [
    (1, 1, 8, 2, 30001, 1, torch.bfloat16),         # about sixty blocks per item, joined by a launch of their own
    (1, 1, 14, 2, 9000, 4, torch.float32),          # 28 rows
    (1, 2, 12, 2, 5003, 9, torch.float16),          # 54 rows: two warps of them
    (1, 1, 10, 2, 6000, 30, torch.float32),         # two row tiles, 25 tokens and 5
    (1, 1, 16, 4, 9001, 100, torch.bfloat16),       # four row tiles
])
def test_chunk_of_few_rows_over_a_long_cache(L, B, Hq, Hkv, context, T, dtype):
    g = gen(L + B + Hq + context)
    n = context + T
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        v = randn(g, L, B, Hkv, n, D)
        if T > 1:
            v[..., n - 1, 3] = math.inf             # only the last token sees it
        e, k, v = loaded(g, L, B, Hq, Hkv, n, v=v, weights=True, stream=stream)
        q = randn(g, L, B, T, Hq, D)
        out = run_chunk(e, q, dtype, weights=binding.WEIGHTS_SET)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(run_chunk(e, q, dtype, weights=binding.WEIGHTS_SET)))
        if T > 1:
            assert not bool(torch.isfinite(out[:, :, -1, :, 3]).any())
        ref, size, weights = chunk_ref(q, k, v, T)
        assert_chunk(out, ref, size, e.state_views()["weights"][:, :n], weights)
        before, again, graph = e.state_views()["weights"][:, :n].clone(), torch.empty_like(out), torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            e.attend_chunk(q, again, weights=binding.WEIGHTS_ADD)
        for _ in range(2):
            graph.replay()
        e.synchronize()
        assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(out))
        # x = sum / G is rounded by the first call (1 step u = 2^-24 of x), and added unrounded by the others (rounded at 2 x and 3 x): 6 u x off
        # 3 x; three times the first is 3 u x off, and 5 u x more by its own two additions: 14 u x between them, below 15 of `before`
        three = before.double() * 3
        assert bool(((e.state_views()["weights"][:, :n].double() - three).abs() <= 15 * 2.0 ** -24 * before.double()).all())


@pytest.mark.parametrize("L,B,P,Hq,Hkv,N,context,T", [
    (1, 2, 1, 8, 2, 1, 0, 1),
    (1, 4, 2, 28, 4, 127, 5, 30),
    (2, 6, 3, 6, 6, 128, 0, 140),
    (1, 3, 1, 9, 3, 129, 100, 43),
    (1, 2, 1, 5, 1, 9001, 60, 7),                              # many blocks per item
    (1, 4, 1, 16, 2, 700, 300, 200),
])
def test_chunk_behind_a_prefix(L, B, P, Hq, Hkv, N, context, T):
    g = gen(N)
    pre, kp, vp = loaded(g, L, P, Hq, Hkv, N)
    e = engine(L, Hq, Hkv, B, context + T, weights=True)
    e.set_page_table(np.random.RandomState(T).permutation(e.info().units * e.info().pages_per_unit))
    e.attach_prefix(pre)
    k, v = randn(g, L, B, Hkv, context + T, D), randn(g, L, B, Hkv, context + T, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    q = randn(g, L, B, T, Hq, D)
    out, size, w = chunk_ref(q, k, v, T, kp, vp)
    got = run_chunk(e, q, weights=binding.WEIGHTS_SET)
    assert_chunk(got, out, size, e.state_views()["weights"][:, :context + T], w)


@pytest.mark.parametrize("order", [1, -1])
def test_chunk_with_references_that_have_to_rise(order):
    """Keys that grow (or shrink) along the cache: the running maximum moves by orders of magnitude."""
    g = gen(5)
    L, B, Hq, Hkv, n, T = 1, 2, 8, 2, 1500, 200
    k = randn(g, L, B, Hkv, n, D)
    grow = torch.linspace(0.01, 3.0, n, device="cuda")[::order] if order > 0 else torch.linspace(3.0, 0.01, n, device="cuda")
    k = (k.float() * grow[:, None]).to(torch.bfloat16)
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k, weights=True)
    q = randn(g, L, B, T, Hq, D)
    out, size, w = chunk_ref(q, k, v, T)
    assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), out, size, e.state_views()["weights"][:, :n], w)


def test_chunk_sees_nothing_of_later_tokens_and_stale_slots():
    """NaN and infinities in keys and values behind the last token, and inside the chunk: a row sees those of its own tokens only."""
    g = gen(6)
    L, B, Hq, Hkv = 1, 3, 12, 2
    e = engine(L, Hq, Hkv, B, 400, weights=True)
    for value in (float("nan"), float("inf"), float("-inf")):
        for n, T, at in ((70, 40, 55), (129, 129, 128), (200, 30, 199), (390, 260, 200), (390, 5, 385)):
            e.reset()
            bad = torch.full((L, B, Hkv, 400, D), value, dtype=torch.bfloat16, device="cuda")
            e.prefill(bad, bad)
            e.reset()
            k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, T, Hq, D)
            e.append(k.transpose(2, 3), v.transpose(2, 3))
            out, size, w = chunk_ref(q, k, v, T)
            assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), out, size, e.state_views()["weights"][:, :n], w)
            # one token of the chunk with a value that is not finite
            v[:, 1, :, at, 3::16] = value
            e.reset()
            e.append(k.transpose(2, 3), v.transpose(2, 3))
            out, size, w = chunk_ref(q, k, v, T)
            got = run_chunk(e, q, weights=binding.WEIGHTS_SET)
            assert_chunk(got, out, size, e.state_views()["weights"][:, :n], w)
            assert int((~torch.isfinite(got)).sum()) == (n - at) * Hq * 8       # from that token on
            # and one with such a key: its logits are not finite, those of rows before it are
            k[:, 1, :, at] = value
            e.reset()
            e.append(k.transpose(2, 3), v.transpose(2, 3))
            got = run_chunk(e, q, weights=binding.WEIGHTS_SET)
            first = at - (n - T)
            assert_chunk(got[:, :, :first], out[:, :, :first], size[:, :, :first])
            assert bool(torch.isfinite(got[:, 0]).all())


def test_chunk_of_any_strides_and_a_poisoned_border():
    """Outputs into strided memory leave what lies between alone; queries of layers, sequences and heads in any order."""
    g = gen(7)
    L, B, T, Hq, Hkv, n = 2, 3, 21, 6, 2, 50
    e, k, v = loaded(g, L, B, Hq, Hkv, n)
    q = randn(g, B, Hq, T, L, D).permute(3, 0, 2, 1, 4)        # [L, B, T, Hq, D]
    room = torch.full((T, L, Hq + 2, B, D + 8), 3.0, dtype=torch.float32, device="cuda")
    view = room[:, :, 1:Hq + 1, :, :D].permute(1, 3, 0, 2, 4)
    e.attend_chunk(q, view)
    e.synchronize()
    out, size, _ = chunk_ref(q, k, v, T)
    assert_chunk.dtype = torch.float32
    assert_chunk(view, out, size)
    mask = torch.ones_like(room, dtype=torch.bool)
    mask[:, :, 1:Hq + 1, :, :D] = False
    assert bool((room[mask] == 3.0).all())


def test_chunk_of_one_token_is_attend():
    g = gen(8)
    L, B, Hq, Hkv, n = 2, 3, 28, 4, 1000
    e, k, v = loaded(g, L, B, Hq, Hkv, n, weights=True)
    q, a = randn(g, L, B, 1, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    e.attend(q[:, :, 0], a)
    got = run_chunk(e, q, weights=binding.WEIGHTS_SET)
    out, size, w = chunk_ref(q, k, v, 1)
    assert_chunk(got, out, size, e.state_views()["weights"][:, :n], w)
    assert bool(((a.double() - got[:, :, 0].double()).abs() <= 2.0 ** -7 * out[:, :, 0].abs() + 2.0 ** -7 * size[:, :, 0]).all())
    p = e.state_views()["pbar"][:, :n].double()
    assert bool(((p - w).abs() <= 2.0 ** -12 * w + 1e-30).all())


def test_chunk_over_a_cache_too_long_for_a_decode_step():
    """300 000 tokens, a few rows: the walk is cut across the whole GPU."""
    g = gen(9)
    L, B, Hq, Hkv, n, T = 1, 1, 4, 1, 300001, 2
    e, k, v = loaded(g, L, B, Hq, Hkv, n, weights=True)
    q = randn(g, L, B, T, Hq, D)
    out, size, w = chunk_ref(q, k, v, T)
    assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), out, size, e.state_views()["weights"][:, :n], w)


def test_pages_behind_four_gigabytes():
    g = gen(10)
    L, B, Hq, Hkv, n, T = 1, 1, 8, 4, 500, 60
    e = binding.Engine(L, Hq, Hkv, D, 2 ** 22, 64, 2.0, batch=B, weights=True)        # 65 537 pages per unit
    inf = e.info()
    assert inf.units * inf.pages_per_unit * 32768 > 2 ** 32
    e.set_page_table(np.arange(inf.units * inf.pages_per_unit)[::-1].copy())
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, T, Hq, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    out, size, w = chunk_ref(q, k, v, T)
    assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), out, size, e.state_views()["weights"][:, :n], w)
    check_sparse(e, randn(g, L, B, Hq, D), k, v, 3)
    small = engine(L, Hq, Hkv, B, 200, weights=True)
    e.set_score_mode(binding.SCORE_WEIGHT)
    weights = e.dump_state()
    assert e.evict_to(200, small) == 300
    check_kept(weights, None, small, k, v, e.state_views()["weights"][:, :n].cpu().numpy(), 200, 64, 0)


# ---- weights ------------------------------------------------------------------------------------------------------------

def test_weights_of_chunks_and_steps_add_up():
    """A prompt in three chunks, then decode steps: the weights are the sums of the probabilities, and move with evictions."""
    g = gen(11)
    L, B, Hq, Hkv = 2, 2, 8, 2
    e = binding.Engine(L, Hq, Hkv, D, 150, 16, 2.0, batch=B, n_recent=8, n_initial=2, max_prefill=200, weights=True)
    e.set_score_mode(binding.SCORE_WEIGHT)
    k, v = randn(g, L, B, Hkv, 170, D), randn(g, L, B, Hkv, 170, D)
    total = torch.zeros(L * B * Hkv, 170, dtype=torch.float64, device="cuda")
    for a, b in ((0, 64), (64, 65), (65, 170)):
        e.append(k[:, :, :, a:b].transpose(2, 3), v[:, :, :, a:b].transpose(2, 3))
        q = randn(g, L, B, b - a, Hq, D)
        out, size, w = chunk_ref(q, k[:, :, :, :b], v[:, :, :, :b], b - a)
        total[:, :b] += w
        got = run_chunk(e, q, weights=binding.WEIGHTS_ADD)
        assert_chunk(got, out, size, e.state_views()["weights"][:, :b], total[:, :b])
    out = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    weights = e.state_views()["weights"]
    before = weights[:, :170].clone()
    for step in range(1, 16):
        e.decode_step(*(randn(g, L, B, h, D) for h in (Hq, Hkv, Hkv)), out)
        n = 170 + step
        # float32 sums, in the order they are made
        want = torch.cat((before, torch.zeros(L * B * Hkv, 1, device="cuda")), 1) + e.state_views()["pbar"][:, :n]
        assert torch.equal(weights[:, :n], want)
        before = want.clone()
    e.attend(randn(g, L, B, Hq, D), out)
    assert torch.equal(weights[:, :185], before)               # (asking again adds nothing)
    snap = e.dump_state(score=True, kv=True)
    assert np.array_equal(snap["score"], before.double().cpu().numpy())
    # the 16th step evicts, by weights that count it
    q, kn, vn = (randn(g, L, B, h, D) for h in (Hq, Hkv, Hkv))
    fork = binding.Engine(L, Hq, Hkv, D, 150, 16, 2.0, batch=B, n_recent=8, n_initial=2, max_prefill=200, weights=True)
    fork.set_auto_evict(False)
    fork.copy_state_from(e)
    fork.decode_step(q, kn, vn, out)
    full = fork.state_views()["weights"][:, :186].cpu().numpy()
    whole = fork.dump_state(kv=True)
    e.decode_step(q, kn, vn, out)
    assert e.info().n == 150
    check_kept(whole, None, e, None, None, full, 150, 8, 2, state=whole)
    # a snapshot brings the weights back
    back = binding.Engine(L, Hq, Hkv, D, 150, 16, 2.0, batch=B, n_recent=8, n_initial=2, max_prefill=200, weights=True)
    back.set_score_mode(binding.SCORE_WEIGHT)
    back.load_state(snap, 170)
    assert torch.equal(back.state_views()["weights"][:, :185], before)
    back.decode_step(q, kn, vn, out)
    a, b = e.dump_state(kv=True, score=True), back.dump_state(kv=True, score=True)
    assert all(np.array_equal(a[x], b[x]) for x in ("pos", "ts", "mri", "score", "k", "v"))


def test_weights_begin_at_zero_again():
    g = gen(12)
    e, k, v = loaded(g, 1, 1, 4, 1, 100, weights=True)
    run_chunk(e, randn(g, 1, 1, 100, 4, D), weights=binding.WEIGHTS_SET)
    assert bool((e.state_views()["weights"][:, :100] > 0).all())
    e.reset()
    e.append(k.transpose(2, 3)[:, :, :60], v.transpose(2, 3)[:, :, :60])
    assert not bool(e.state_views()["weights"][:, :60].any())
    out = torch.empty(1, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    e.decode_step(randn(g, 1, 1, 4, D), randn(g, 1, 1, 1, D), randn(g, 1, 1, 1, D), out)
    assert torch.equal(e.state_views()["weights"][:, :61], e.state_views()["pbar"][:, :61])
    e.reset()
    q = randn(g, 30, 1, 1, 4, D)
    e.prefill_observed(q, k[:, :, :, :30].contiguous(), v[:, :, :, :30].contiguous(), torch.empty_like(q))
    assert not bool(e.state_views()["weights"][:, :30].any())


# ---- eviction by weight and into another cache ------------------------------------------------------------------------------

def kept_slots(w, n, keep, R, S):
    """The rule, token by token: what is no number first, then by weight, of equals the more recent."""
    middle = sorted(range(S, n - R), key=lambda i: (not math.isnan(w[i]), 0.0 if math.isnan(w[i]) else -w[i], -i))[:keep - S - R]
    return np.array(sorted(list(range(S)) + middle + list(range(n - R, n))))


def check_kept(before, _, dst, k, v, w, keep, R, S, state=None):
    n = w.shape[1]
    d = dst.dump_state(kv=True)
    assert d["n"] == keep
    for u in range(w.shape[0]):
        at = kept_slots(w[u], n, keep, R, S)
        assert np.array_equal(d["pos"][u], before["pos"][u][at])
        assert np.array_equal(d["ts"][u], before["ts"][u][at]) and np.array_equal(d["mri"][u], before["mri"][u][at])
        if state is not None:
            assert np.array_equal(d["k"][u], state["k"][u][at]) and np.array_equal(d["v"][u], state["v"][u][at])
        else:
            for x, y in (("k", k), ("v", v)):
                assert np.array_equal(d[x][u].view(np.int16), y.flatten(0, 2)[u].cpu().view(torch.int16).numpy()[at])
        got = dst.state_views()["weights"][u, :keep].cpu().numpy()
        assert np.array_equal(got, w[u][at], equal_nan=True)


@pytest.mark.parametrize("L,B,Hkv,n,keep,R,S,kind", [
    (1, 1, 1, 2, 1 + 1, 1, 0, "normal"),           # all of them
    (1, 1, 1, 3, 2, 1, 0, "normal"),
    (2, 3, 2, 65, 64, 5, 3, "normal"),
    (1, 2, 2, 700, 250, 32, 4, "heavy"),
    (1, 2, 2, 700, 250, 32, 4, "zero"),            # all alike: the more recent
    (1, 2, 2, 700, 250, 32, 4, "few"),             # more are kept than have any weight
    (1, 2, 2, 700, 250, 32, 4, "coarse"),          # many equal ones at the cut
    (1, 2, 2, 700, 250, 32, 4, "nan"),
    (1, 2, 2, 1500, 1400, 1, 0, "heavy"),
    (1, 1, 2, 50000, 1001, 3, 17, "heavy"),        # keys that do not fit shared memory
    (1, 1, 2, 50000, 40000, 3, 17, "coarse"),
    (1, 1, 2, 41000, 77, 40, 0, "few"),
])
def test_evict_by_weight(L, B, Hkv, n, keep, R, S, kind):
    g = gen(n + keep)
    units = L * B * Hkv
    e, k, v = loaded(g, L, B, 2 * Hkv, Hkv, n, weights=True, n_recent=R, n_initial=S, window=max(R, 1))
    e.set_score_mode(binding.SCORE_WEIGHT)
    w = torch.randn(units, n, generator=g, device="cuda")
    w = {"normal": w.abs(), "heavy": torch.exp(3 * w), "zero": w * 0, "few": torch.where(w > 2.5, w, 0.0), "coarse": (w.abs() * 2).round() / 2,
         "nan": torch.where(w > 1.8, float("nan"), w)}[kind]
    e.state_views()["weights"][:, :n] = w
    e.state_views()["ts_mri"][:, :n] = torch.randint(0, 9, (units, n, 2), generator=g, device="cuda", dtype=torch.int32)
    before, w = e.dump_state(), w.cpu().numpy()
    small = engine(L, 2 * Hkv, Hkv, B, keep, weights=True)
    small.set_page_table(np.random.RandomState(n).permutation(small.info().units * small.info().pages_per_unit))
    evictions = e.info().evictions
    assert e.evict_to(keep, small) == n - keep
    assert e.info().n == n and e.info().evictions == evictions and small.info().next_position == e.info().next_position
    check_kept(before, None, small, k, v, w, keep, R, S)
    assert e.evict_to(keep) == n - keep                        # and in place
    check_kept(before, None, e, k, v, w, keep, R, S)
    assert e.evict_to(keep) == 0
    if keep < n:
        assert e.info().evictions == evictions + 1
    # both go on alike
    q, kn, vn = randn(g, L, B, 2 * Hkv, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
    a, b = torch.empty_like(q), torch.empty_like(q)
    e.decode_step(q, kn, vn, a)
    small.decode_step(q, kn, vn, b)
    x, y = e.dump_state(kv=True), small.dump_state(kv=True)
    assert torch.equal(a, b) and all(np.array_equal(x[i], y[i]) for i in ("pos", "ts", "mri", "k", "v"))


@pytest.mark.parametrize("mode", [0, 1, 2, 3])
def test_evict_to_by_the_papers_scores(mode):
    """At once, into another handle: what the lagged eviction keeps at the same step."""
    g = gen(40 + mode)
    L, B, Hq, Hkv, W = 1, 2, 8, 2, 16
    make = lambda: binding.Engine(L, Hq, Hkv, D, 64, W, 0.02, batch=B, max_prefill=100)
    a, b, c = make(), make(), make()
    k, v = randn(g, L, B, Hkv, 100, D), randn(g, L, B, Hkv, 100, D)
    out = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    for e in (a, b):
        e.set_score_mode(mode)
        e.set_auto_evict(False)
        e.prefill(k, v)
    for _ in range(W):
        q, kn, vn = (randn(g, L, B, h, D) for h in (Hq, Hkv, Hkv))
        for e in (a, b):
            e.decode_step(q, kn, vn, out)
    assert b.evict_to(64, c) == 100 + W - 64 and a.evict() == 100 + W - 64
    assert b.info().n == 100 + W and c.info().t == W
    assert b.evict_to(64) == 100 + W - 64
    x, y, z = (e.dump_state(kv=True) for e in (a, b, c))
    for i in ("pos", "ts", "mri", "k", "v"):
        assert np.array_equal(x[i], y[i]) and np.array_equal(x[i], z[i])


def test_evict_to_copies_short_caches_whole_between_streams_and_without_weights():
    g = gen(13)
    s0, s1 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    a, b = engine(1, 8, 2, 3, 500, stream=s0, weights=True), engine(1, 8, 2, 3, 300, stream=s1)
    a.set_score_mode(binding.SCORE_WEIGHT)
    k, v = randn(g, 1, 3, 2, 400, D), randn(g, 1, 3, 2, 400, D)
    torch.cuda.synchronize()
    a.prefill(k, v)
    with torch.cuda.stream(s0):
        a.state_views()["weights"][:, :400] = torch.arange(400, 0, -1, device="cuda", dtype=torch.float32)
    assert a.evict_to(300, b) == 100
    a.reset()                                                  # right behind: the rows have moved before
    a.prefill(torch.zeros_like(k), torch.zeros_like(v))
    at = np.concatenate((np.arange(299), [399]))
    d = b.dump_state(kv=True)
    assert np.array_equal(d["pos"], np.tile(at, (6, 1)))
    assert np.array_equal(d["k"].view(np.int16), k.flatten(0, 2).cpu().view(torch.int16).numpy()[:, at])
    c = engine(1, 8, 2, 3, 300, weights=True)
    assert b.evict_to(300, c) == 0                             # (b holds 300: all of them)
    x = c.dump_state(kv=True)
    assert all(np.array_equal(x[i], d[i]) for i in ("pos", "ts", "mri", "k", "v")) and not bool(c.state_views()["weights"][:, :300].any())


# ---- selected blocks ------------------------------------------------------------------------------------------------------

def sparse_ref(q, k, v, blocks, kp=None, vp=None):
    """out, sum p |v|, the selected blocks [units, blocks]."""
    L, B, Hq, _ = q.shape
    Hkv, n = k.shape[2:4]
    G, last = Hq // Hkv, (n - 1) // 64
    picked = min(blocks - 1, last)
    out, size = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape, dtype=torch.float64, device="cuda")
    chosen = np.full((L, B, Hkv, blocks), -1, np.int32)
    for l in range(L):
        for b in range(B):
            for h in range(Hkv):
                kk, vv, qq = k[l, b, h].double(), v[l, b, h].double(), q[l, b, h * G:(h + 1) * G].double()
                full = kk[:last * 64].view(last, 64, D)
                hi, lo = full.amax(1), full.amin(1)
                s = torch.maximum(hi[:, None] * qq, lo[:, None] * qq).sum((1, 2)).cpu().numpy()
                order = sorted(range(last), key=lambda i: (not math.isnan(s[i]), 0.0 if math.isnan(s[i]) else -s[i], i))[:picked]
                chosen[l, b, h, :picked + 1] = sorted(order) + [last]
                at = torch.cat([torch.arange(c * 64, min(n, c * 64 + 64), device="cuda") for c in chosen[l, b, h, :picked + 1]])
                kk, vv = kk[at], vv[at]
                if kp is not None:
                    p = b // (B // kp.shape[1])
                    kk, vv = torch.cat((kp[l, p, h].double(), kk)), torch.cat((vp[l, p, h].double(), vv))
                p = torch.softmax(qq @ kk.T / math.sqrt(D), -1)
                out[l, b, h * G:(h + 1) * G], size[l, b, h * G:(h + 1) * G] = p @ vv, p @ vv.abs()
    return out, size, chosen.reshape(-1, blocks)


def check_sparse(e, q, k, v, blocks, kp=None, vp=None):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    sel = torch.full((e.info().units, blocks), 99, dtype=torch.int32, device="cuda")
    pbar = e.state_views()["pbar"].clone()
    e.attend_sparse(q, out, blocks, sel)
    e.synchronize()
    ref, size, chosen = sparse_ref(q, k, v, blocks, kp, vp)
    assert np.array_equal(sel.cpu().numpy(), chosen)
    err, tol = (out.double() - ref).abs(), 2.0 ** -8 * ref.abs() + 2.0 ** -13 * size + 1e-30
    assert torch.equal(torch.isfinite(out), torch.isfinite(ref)) and bool((err <= tol)[torch.isfinite(ref)].all())
    assert torch.equal(e.state_views()["pbar"], pbar)
    other = torch.empty_like(out)
    e.attend_sparse(q, other, blocks)
    assert torch.equal(out, other) or not bool(torch.isfinite(ref).all())
    return out


@pytest.mark.parametrize("L,B,Hq,Hkv,n,blocks", [
    (1, 1, 1, 1, 1, 1), (1, 1, 8, 2, 64, 3), (1, 2, 8, 2, 65, 1), (1, 2, 8, 2, 65, 2), (1, 2, 8, 2, 128, 1),
    (2, 3, 28, 4, 1000, 5), (2, 3, 6, 6, 1001, 15), (1, 2, 9, 3, 1001, 16), (1, 2, 40, 8, 1001, 17), (1, 2, 16, 2, 4097, 64),
    (1, 1, 8, 2, 70001, 3), (1, 1, 4, 1, 140000, 1100),     # too long for a decode step; many blocks
    (5, 70, 4, 2, 200, 2),
])
def test_sparse_against_64_bits(L, B, Hq, Hkv, n, blocks):
    g = gen(n + blocks)
    e, k, v = loaded(g, L, B, Hq, Hkv, n)
    check_sparse(e, randn(g, L, B, Hq, D), k, v, blocks)
    if n > 64:                                                 # the bounds as they are laid out
        last = (n - 1) // 64
        rows = k.flatten(0, 2)[:, :last * 64].unflatten(1, (last, 64))
        got = e.block_bounds()[:, :last]
        assert torch.equal(got[:, :, 0], rows.amax(2)) and torch.equal(got[:, :, 1], rows.amin(2))


def test_sparse_ties_go_to_the_older_block_and_all_blocks_are_attend():
    g = gen(14)
    L, B, Hq, Hkv, n = 1, 2, 8, 2, 64 * 40 + 7
    one = randn(g, L, B, Hkv, 64, D)
    k = torch.cat((one.repeat(1, 1, 1, 40, 1), one[:, :, :, :7]), 3).contiguous()
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k)
    q = randn(g, L, B, Hq, D)
    sel = torch.empty(L * B * Hkv, 9, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, torch.empty_like(q), 9, sel)
    assert sel.cpu().tolist() == [list(range(8)) + [40]] * 4
    a, b = torch.empty_like(q), torch.empty_like(q)
    e.attend(q, a)
    for blocks in (41, 42, 1000):
        e.attend_sparse(q, b, blocks)
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [64 * 200 + 3, 64 * 700 + 3])       # scored by a unit's own block of threads, by many
@pytest.mark.parametrize("kind", ["no queries", "close", "many close", "far apart", "infinite", "negative"])
def test_sparse_scores_near_the_cut(n, kind):
    """Blocks whose scores are equal, closer than float32 tells apart, or of very different size: the choice is that of 64 bits."""
    g = gen(23)
    L, B, Hq, Hkv, blocks = 1, 2, 8, 2, 70
    last = (n - 1) // 64
    k = randn(g, L, B, Hkv, n, D)
    q = randn(g, L, B, Hq, D)
    if kind == "no queries":
        q.zero_()
    elif kind in ("close", "many close"):
        # large equal parts and differences of 2^-30 of them in one dimension
        k[:] = 0
        k[..., 0] = 256.0
        q[:] = 0
        q[..., 0], q[..., 1] = 256.0, 2.0 ** -7
        some = last if kind == "many close" else 100
        step = torch.randint(1, 200, (L, B, Hkv, some), generator=g, device="cuda").to(torch.bfloat16) * 2.0 ** -9
        k[:, :, :, :some * 64, 1] = step.repeat_interleave(64, -1)
        k[:, :, :, some * 64:, 0] = 128.0
    elif kind == "far apart":
        k *= torch.exp(6 * torch.randn(L, B, Hkv, n // 64 + 1, generator=g, device="cuda")).repeat_interleave(64, -1)[..., :n, None].to(torch.bfloat16)
    elif kind == "infinite":
        k[:, :, :, 64 * 5 + 3, 7] = float("inf")
        k[:, :, :, 64 * 9 + 3, 7] = float("-inf")
    else:
        k, q = -k.abs() - 1, q.abs()
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k.contiguous())
    sel = torch.full((L * B * Hkv, blocks), 99, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, torch.empty_like(q), blocks, sel)
    e.synchronize()
    assert np.array_equal(sel.cpu().numpy(), sparse_ref(q, k, v, blocks)[2])


def test_sparse_follows_the_cache():
    """Bounds of blocks that fill while decoding, after an eviction, after a reset, after a fork; pages that a caller has written."""
    g = gen(15)
    L, B, Hq, Hkv = 1, 2, 8, 2
    e = binding.Engine(L, Hq, Hkv, D, 256, 32, 0.05, batch=B, n_recent=16, max_prefill=300)
    out = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    for seed in (1, 2):
        n = 300 if seed == 1 else 100
        e.prefill(*(randn(g, L, B, Hkv, n, D) for _ in range(2)))
        for step in range(70):
            e.decode_step(*(randn(g, L, B, h, D) for h in (Hq, Hkv, Hkv)), out)
            if step % 7 == 0 or step == 31:
                d = e.dump_state(kv=True)
                k, v = (torch.from_numpy(d[x].view(np.int16).copy()).view(torch.bfloat16).view(L, B, Hkv, -1, D).cuda() for x in ("k", "v"))
                check_sparse(e, randn(g, L, B, Hq, D), k, v, 3)
        if seed == 1:
            fork = binding.Engine(L, Hq, Hkv, D, 256, 32, 0.05, batch=B, n_recent=16, max_prefill=300)
            fork.copy_state_from(e)
            d = e.dump_state(kv=True)
            k, v = (torch.from_numpy(d[x].view(np.int16).copy()).view(torch.bfloat16).view(L, B, Hkv, -1, D).cuda() for x in ("k", "v"))
            check_sparse(fork, randn(g, L, B, Hq, D), k, v, 2)
            e.reset()
    # keys written behind the library's back
    view = e.state_views()
    page = int(view["page_table"][0, 0])
    view["pages"][page, 0] *= 3
    d = e.dump_state(kv=True)
    k, v = (torch.from_numpy(d[x].view(np.int16).copy()).view(torch.bfloat16).view(L, B, Hkv, -1, D).cuda() for x in ("k", "v"))
    e.index_blocks(0)
    check_sparse(e, randn(g, L, B, Hq, D), k, v, 2)


def test_sparse_behind_a_prefix():
    g = gen(16)
    L, B, P, Hq, Hkv, N, n = 2, 4, 2, 28, 4, 200, 500
    pre, kp, vp = loaded(g, L, P, Hq, Hkv, N)
    e = engine(L, Hq, Hkv, B, n)
    e.attach_prefix(pre)
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    for blocks in (1, 4, 50):
        check_sparse(e, randn(g, L, B, Hq, D), k, v, blocks, kp, vp)


def test_sparse_scores_that_are_no_numbers():
    """A block with a NaN or infinite key is read (its rows are what they are in a decode step); stale ones behind the last token are not seen."""
    g = gen(17)
    L, B, Hq, Hkv, n = 1, 1, 4, 1, 700
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, Hq, D)
    k[0, 0, 0, 130, 5] = float("nan")
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k, v=v)
    sel = torch.empty(1, 2, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, torch.empty_like(q), 2, sel)
    assert sel.cpu().tolist() == [[2, 10]]
    bad = torch.full((L, B, Hkv, n, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    e.reset()
    e.prefill(bad, bad)
    e.index_blocks()
    e.reset()
    k, v = randn(g, L, B, Hkv, 333, D), randn(g, L, B, Hkv, 333, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    check_sparse(e, q, k, v, 3)


# ---- calls ---------------------------------------------------------------------------------------------------------------

def test_calls_refuse_bad_arguments():
    g = gen(18)
    L, B, Hq, Hkv, n = 1, 2, 8, 2, 100
    e, k, v = loaded(g, L, B, Hq, Hkv, n)
    lib = binding.lib()
    q, out = randn(g, L, B, 4, Hq, D), torch.empty(L, B, 4, Hq, D, dtype=torch.bfloat16, device="cuda")
    e.reserve_chunk(100)
    space = e._chunk_space[-1].data_ptr()

    def refused(code, *args):
        assert lib.lazyev_attend_chunk(e._h, *args) == code and lib.lazyev_last_error(e._h)

    qi, oi = e._rows(0, q, Hq, 4), e._rows(2, out, Hq, 4)
    refused(binding.EINVAL, qi, 0, oi, 0, space)
    refused(binding.EINVAL, qi, -1, oi, 0, space)
    refused(binding.EINVAL, qi, n + 1, oi, 0, space)
    refused(binding.EINVAL, None, 4, oi, 0, space)
    refused(binding.EINVAL, qi, 4, None, 0, space)
    refused(binding.EINVAL, qi, 4, oi, 3, space)
    refused(binding.ESTATE, qi, 4, oi, binding.WEIGHTS_SET, space)
    refused(binding.EINVAL, qi, 4, oi, 0, None)
    refused(binding.EINVAL, qi, 4, oi, 0, space + 128)
    for bad in (q.float(), q.half()):                          # queries of other types
        with pytest.raises(binding.LazyEvError) as err:
            e.attend_chunk(bad, out)
        assert err.value.code == binding.EINVAL
    for bad in (q[:, :, :1].expand(L, B, 4, Hq, D), q.flip(2)[:, :, :, :1].expand(L, B, 4, Hq, D)):       # repeated rows
        with pytest.raises(binding.LazyEvError) as err:
            e.attend_chunk(bad, out)
        assert err.value.code == binding.EINVAL
    with pytest.raises(binding.LazyEvError) as err:            # overlapping outputs
        e.attend_chunk(q, out[:, :, :1].expand(L, B, 4, Hq, D))
    assert err.value.code == binding.EINVAL
    for args in ((q[..., :7, :], out), (q, out[:, :, :3]), (q.transpose(3, 4), out), (q[:, :1], out), (None, out), (q, None), (q[:, :, :0], out[:, :, :0])):
        with pytest.raises((ValueError, binding.LazyEvError)):
            e.attend_chunk(*args)
    with pytest.raises(ValueError):
        e.attend_chunk(q.cpu(), out)
    # eviction into another handle
    def evict_refused(code, keep, dst=None):
        with pytest.raises(binding.LazyEvError) as err:
            e.evict_to(keep, dst)
        assert err.value.code == code

    evict_refused(binding.EINVAL, 1)                           # (one recent token is protected)
    evict_refused(binding.EINVAL, e.info().budget + 1)
    evict_refused(binding.EINVAL, 50, engine(L, Hq, Hkv, B + 1, 60))
    evict_refused(binding.EINVAL, 50, engine(L, 12, Hkv, B, 60))
    evict_refused(binding.ESTATE, 50, loaded(g, L, B, Hq, Hkv, 60)[0])
    evict_refused(binding.ECAPACITY, 90, engine(L, Hq, Hkv, B, 20))
    other = engine(L, Hq, Hkv, B, 60)
    other.attach_prefix(e)
    evict_refused(binding.ESTATE, 50, other)                   # another prefix
    evict_refused(binding.ESTATE, 50)                          # in place under a handle that shares it
    other.detach_prefix()
    assert e.info().n == n
    with pytest.raises(binding.LazyEvError) as err:
        engine(L, Hq, Hkv, B, 60).evict_to(20)
    assert err.value.code == binding.ESTATE
    # blocks
    q1, o1 = q[:, :, 0].contiguous(), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    assert lib.lazyev_attend_sparse(e._h, q1.data_ptr(), 2, o1.data_ptr(), None) == binding.ESTATE       # no workspace yet
    assert lib.lazyev_index_blocks(e._h, 0) == binding.ESTATE
    assert lib.lazyev_set_block_workspace(e._h, 64) == binding.EINVAL
    e.index_blocks()
    for args in ((None, 2, o1.data_ptr(), None), (q1.data_ptr(), 0, o1.data_ptr(), None), (q1.data_ptr(), 2, None, None),
                 (q1.data_ptr() + 8, 2, o1.data_ptr(), None), (q1.data_ptr(), 2, o1.data_ptr() + 1, None), (q1.data_ptr(), 2, o1.data_ptr(), 2)):
        assert lib.lazyev_attend_sparse(e._h, *args) == binding.EINVAL
    assert lib.lazyev_index_blocks(e._h, -1) == binding.EINVAL
    with pytest.raises(ValueError):
        e.attend_sparse(q1, o1, 2, torch.empty(4, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        e.attend_sparse(q, o1, 2)
    empty = engine(L, Hq, Hkv, B, 60)
    with pytest.raises(binding.LazyEvError) as err:
        empty.attend_sparse(q1, o1, 2)
    assert err.value.code == binding.ESTATE
    with pytest.raises(binding.LazyEvError) as err:
        empty.copy_state_from(loaded(g, L, B, Hq, Hkv, 60, weights=True)[0])
    assert err.value.code == binding.EINVAL
    assert_chunk.dtype = torch.bfloat16
    ref, size, _ = chunk_ref(q, k, v, 4)
    assert_chunk(run_chunk(e, q), ref, size)                   # nothing of it changed anything


def test_captured_and_replayed_on_a_stream_of_its_own():
    g = gen(19)
    L, B, Hq, Hkv, n, T = 1, 3, 8, 2, 1500, 40
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        e, k, v = loaded(g, L, B, Hq, Hkv, n, weights=True, stream=stream)
        q, out = randn(g, L, B, T, Hq, D), torch.empty(L, B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
        q1, o1 = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
        sel = torch.empty(L * B * Hkv, 4, dtype=torch.int32, device="cuda")
        e.reserve_chunk(T, binding.WEIGHTS_SET)
        e._blocks()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):           # (the first call of all: the bounds are made inside)
            e.attend_chunk(q, out, weights=binding.WEIGHTS_SET)
            e.attend_sparse(q1, o1, 4, sel)
        e.attend_sparse(randn(g, L, B, Hq, D), torch.empty_like(o1), 4)        # and an eager one before the first replay
        for seed in (1, 2):
            q.copy_(randn(gen(seed), L, B, T, Hq, D))
            q1.copy_(randn(gen(seed), L, B, Hq, D))
            graph.replay()
            stream.synchronize()
            ref, size, w = chunk_ref(q, k, v, T)
            assert_chunk.dtype = torch.bfloat16
            assert_chunk(out, ref, size, e.state_views()["weights"][:, :n], w)
            ref, size, chosen = sparse_ref(q1, k, v, 4)
            assert np.array_equal(sel.cpu().numpy(), chosen)
            assert bool(((o1.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -13 * size).all())
        e.synchronize()


@pytest.mark.parametrize("B,context,T,tiles", [(1, 6000, 4, 0), (1, 6000, 4, 1), (40, 700, 200, 0), (40, 700, 200, 3)])
def test_a_chunk_that_starves_reports_and_recovers(B, context, T, tiles):
    """The producers stop after some key tiles: bounded waits run out, the status word tells, and after a reset the handle works again."""
    g = gen(20)
    e, k, v = loaded(g, 1, B, 8, 2, context + T, weights=True)
    q = randn(g, 1, B, T, 8, D)
    out = torch.empty_like(q)
    e.set_wait_limit(0.002)
    e.debug_starve_page_ring(tiles)
    e.attend_chunk(q, out, weights=binding.WEIGHTS_SET)
    with pytest.raises(binding.LazyEvError) as err:
        e.synchronize()
    assert err.value.code == binding.EDEVICE
    e.debug_starve_page_ring(-1)
    e.set_wait_limit(2.0)
    e.reset()
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    ref, size, w = chunk_ref(q, k, v, T)
    assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), ref, size, e.state_views()["weights"][:, :context + T], w)


def test_range_checked_build():
    """The same tests through the build whose kernels check every slot, page and work index."""
    import os
    import subprocess
    import sys
    if binding.debug_bounds_requested():
        pytest.skip("already inside the range-checked run")
    res = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-m", "gpu", "-k",
                          "64_bits or prefix or add_up or by_weight or follows or serving"],
                         env=dict(os.environ, LAZYEV_DEBUG_BOUNDS="1"), capture_output=True, text=True,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-2000:]
    assert " passed" in res.stdout and "failed" not in res.stdout


# ---- together ------------------------------------------------------------------------------------------------------------

def test_serving_run_from_a_long_prompt_to_a_small_cache():
    """A prompt from projected rows in chunks, each attending as it is read and weighing what it sees; the heaviest tokens go on in a
    small cache, which decodes with its weights across evictions, checks drafted tokens in one go and reads selected blocks.  Every
    attention is held to the 64-bit form over the rows that the cache holds."""
    g = gen(21)
    L, B, Hq, Hkv, N = 2, 2, 14, 2, 777
    f, eps = freqs(64, 5e5), 1e-6
    qw, kw = (torch.rand(L, D, generator=g, device="cuda") + 0.5 for _ in range(2))
    big = engine(L, Hq, Hkv, B, N, weights=True, n_recent=32, n_initial=4, window=32)
    small = binding.Engine(L, Hq, Hkv, D, 320, 32, 2.0, batch=B, n_recent=32, n_initial=4, weights=True)
    for e in (big, small):
        e.set_score_mode(binding.SCORE_WEIGHT)
        e.set_rope(f)
        e.set_head_norm(qw, kw, eps)
    qkv = randn(g, L, B, N, Hq + 2 * Hkv, D)
    total = torch.zeros(L * B * Hkv, N, dtype=torch.float64, device="cuda")
    assert_chunk.dtype = torch.bfloat16

    def rows_of(e):
        d = e.dump_state(kv=True)
        return (d, *(torch.from_numpy(d[x].view(np.int16).copy()).view(torch.bfloat16).view(L, B, Hkv, -1, D).cuda() for x in ("k", "v")))

    def turned(x, at):
        q = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
        (big if at < N else small).norm_rope(x, None, q, None, first_position=at)
        return q

    for a, b in ((0, 300), (300, 556), (556, N)):
        rows = qkv[:, :, a:b]
        big.append(rows[..., Hq:Hq + Hkv, :], rows[..., Hq + Hkv:, :])
        q = turned(rows[..., :Hq, :], a)
        _, k, v = rows_of(big)
        out, size, w = chunk_ref(q, k, v, b - a)
        total[:, :b] += w
        got = run_chunk(big, q, weights=binding.WEIGHTS_ADD)
        assert_chunk(got, out, size, big.state_views()["weights"][:, :b], total[:, :b])
    ref, scale = rows_ref(qkv[..., Hq:Hq + Hkv, :], kw, eps, [np.arange(N)] * B, f)
    assert_rows(k.transpose(2, 3).cpu(), ref, scale, torch.bfloat16)

    before, weights = big.dump_state(kv=True), big.state_views()["weights"][:, :N].cpu().numpy()
    assert big.evict_to(300, small) == N - 300
    check_kept(before, None, small, None, None, weights, 300, 32, 4, state=before)

    out = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    evictions = 0
    for step in range(1, 70):
        x = randn(g, L, B, Hq + 2 * Hkv, D)
        at = small.info().next_position
        assert at == N + step - 1
        before, w = small.dump_state(kv=True), small.state_views()["weights"][:, :small.info().n].cpu().numpy()
        q = turned(x[:, :, None, :Hq], at)
        small.decode_step_rows(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], out)
        d, k, v = rows_of(small)
        if d["n"] == before["n"] + 1:
            o, size, p = chunk_ref(q, k, v, 1)
            assert bool(((out.double() - o[:, :, 0]).abs() <= 2.0 ** -8 * o[:, :, 0].abs() + 2.0 ** -13 * size[:, :, 0]).all())
            pbar = small.state_views()["pbar"][:, :d["n"]].cpu().numpy()
            assert np.array_equal(small.state_views()["weights"][:, :d["n"]].cpu().numpy(), np.pad(w, ((0, 0), (0, 1))) + pbar)
        else:
            evictions += 1
            assert d["n"] == 320 and np.all(d["pos"][:, -32:] == np.arange(at - 31, at + 1)) and np.all(d["pos"][:, :4] == before["pos"][:, :4])
        if step % 20 == 0:
            check_sparse(small, turned(x[:, :, None, :Hq], at)[:, :, 0].contiguous(), k, v, 3)
    assert evictions == 2 and small.info().n == 325
    # five drafted tokens, checked in one go
    rows = randn(g, L, B, 5, Hq + 2 * Hkv, D)
    at = small.info().next_position
    small.append(rows[..., Hq:Hq + Hkv, :], rows[..., Hq + Hkv:, :])
    q = turned(rows[..., :Hq, :], at)
    _, k, v = rows_of(small)
    o, size, _ = chunk_ref(q, k, v, 5)
    assert_chunk(run_chunk(small, q), o, size)
