"""Calls on a whole cache at their edges: block scores of infinite and of tiny values, walks and branches that only long caches or
many units reach, weights of every kind of decode step, caches behind a prefix, refusals that leave everything as it was.

Tolerances are those of test_gpu_whole_cache.py where nothing else is said."""
import math

import numpy as np
import pytest
import torch

from paper_2506_15969_b200 import binding
from tests.test_gpu_operators import TYPES, engine, gen, randn
from tests.test_gpu_whole_cache import assert_chunk, check_kept, check_sparse, chunk_ref, loaded, run_chunk, sparse_ref

pytestmark = pytest.mark.gpu

D = 128


# ---- selected blocks --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [64 * 200 + 3, 64 * 700 + 3])       # scored by a unit's own block of threads, by many
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (6, 2)])              # one head, a group of one sign
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("sign", [1, -1, 0, 2])
def test_an_infinite_key_scores_by_its_sign(n, Hq, Hkv, value, sign):
    """max(q high, q low) with high = inf is q low for a negative q, however many heads are negative; for q = 0 it is no number."""
    g = gen(31)
    L, B, blocks = 1, 2, 70
    k, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hq, D)
    for block, d in ((5, 7), (9, 100), (150, 7)):
        k[:, :, :, 64 * block + 3, d] = value
        q[..., d] = sign * (q[..., d].abs() + 0.125)
        if sign == 2:                                                 # (one head of the first group is at zero)
            q[:, :, 0, d] = 0
    k[:, 0, :, 64 * 11:64 * 12, 30] = value                           # a block with no other key in that dimension
    q[..., 30] = q[..., 30].abs() + 0.125
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k)
    sel = torch.full((L * B * Hkv, blocks), 99, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, torch.empty_like(q), blocks, sel)
    e.synchronize()
    assert np.array_equal(sel.cpu().numpy(), sparse_ref(q, k, v, blocks)[2])


@pytest.mark.parametrize("n", [64 * 200 + 3, 64 * 700 + 3])
@pytest.mark.parametrize("k_size,q_size", [(2.0 ** -76, 2.0 ** -71), (2.0 ** -126, 2.0 ** -24), (2.0 ** -60, 2.0 ** -85)])
def test_scores_of_tiny_values_are_those_of_64_bits(n, k_size, q_size):
    """Products that 32 bits hold as a few steps, or not at all."""
    g = gen(32)
    L, B, Hq, Hkv, blocks = 1, 2, 8, 2, 70
    k, q = (randn(g, L, B, Hkv, n, D).double() * k_size).to(torch.bfloat16), (randn(g, L, B, Hq, D).double() * q_size).to(torch.bfloat16)
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k)
    sel = torch.full((L * B * Hkv, blocks), 99, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, torch.empty_like(q), blocks, sel)
    e.synchronize()
    assert np.array_equal(sel.cpu().numpy(), sparse_ref(q, k, v, blocks)[2])


@pytest.mark.parametrize("kind", ["normal", "alike", "two values"])
def test_more_blocks_than_shared_memory_holds_scores_of(kind):
    """Over a million tokens: the scores of a unit stay in device memory, and every way to the cut rewrites them there."""
    g = gen(33)
    L, B, Hq, Hkv, n = 1, 1, 4, 1, 64 * 16390 + 5
    k = randn(g, L, B, Hkv, n, D)
    if kind != "normal":
        k = k[:, :, :, :64].repeat(1, 1, 1, n // 64 + 1, 1)[:, :, :, :n].contiguous()
    if kind == "two values":
        k[:, :, :, 64 * 9000:64 * 9100] *= 2
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k)
    for blocks in (3, 77, 300):
        check_sparse(e, randn(g, L, B, Hq, D), k, v, blocks)


def test_many_units_with_more_blocks_than_shared_memory_holds_scores_of():
    """The same with enough units for a block of threads each: bounds laid down by the caller, every key and value of a unit alike."""
    g = gen(34)
    L, B, Hq, Hkv, n, blocks = 1, 80, 1, 1, 64 * 16386 + 1, 40
    last = n // 64
    e = engine(L, Hq, Hkv, B, n)
    one = randn(g, L, B, 1, Hkv, D)
    e.append(one.expand(L, B, n, Hkv, D), one.expand(L, B, n, Hkv, D))
    e.index_blocks()
    assert torch.equal(e.block_bounds()[:, :last, 0], one.view(B, 1, D).expand(B, last, D))
    low = randn(g, B, last, D)
    high = torch.maximum(low, randn(g, B, last, D))
    e.block_bounds()[:, :last, 0], e.block_bounds()[:, :last, 1] = high, low
    q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    sel = torch.full((B, blocks), 99, dtype=torch.int32, device="cuda")
    e.attend_sparse(q, out, blocks, sel)
    e.synchronize()
    for u in range(B):
        s = torch.maximum(high[u].double() * q[0, u].double(), low[u].double() * q[0, u].double()).sum(-1).cpu().numpy()
        best = np.lexsort((np.arange(last), -s))[:blocks - 1]
        assert sel[u].tolist() == sorted(best.tolist()) + [last]
    assert bool(((out[:, :, 0].double() - one[:, :, 0, 0].double()).abs() <= (2.0 ** -8 + 2.0 ** -13) * one[:, :, 0, 0].double().abs()).all())


def test_blocks_that_no_decode_launch_holds_are_refused_before_anything_is_queued():
    g = gen(35)
    L, B, Hq, Hkv, n = 1, 1, 8, 2, 140001
    e, k, v = loaded(g, L, B, Hq, Hkv, n)
    q, out = randn(g, L, B, Hq, D), torch.full((L, B, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.LazyEvError) as err:                   # (nor does a dense step have a launch shape)
        e.attend(q, out)
    assert err.value.code == binding.EINVAL
    sel = torch.full((L * B * Hkv, 2200), 99, dtype=torch.int32, device="cuda")
    launches = e.info().launches
    with pytest.raises(binding.LazyEvError) as err:
        e.attend_sparse(q, out, 2200, sel)
    assert err.value.code == binding.EINVAL
    e.synchronize()
    assert e.info().launches == launches and bool((sel == 99).all()) and bool((out == 7).all())
    check_sparse(e, q, k, v, 40)


def test_steps_that_append_a_token_and_read_selected_blocks():
    """The step that saves something: no dense pass before it.  t, what is tracked and the weights stay as they are, a new token's weight is 0,
    and no eviction comes due by itself."""
    g = gen(44)
    L, B, Hq, Hkv, n = 1, 2, 8, 2, 190
    e = binding.Engine(L, Hq, Hkv, D, 250, 16, 1e-3, batch=B, n_recent=8, max_prefill=300, weights=True)
    e.set_score_mode(binding.SCORE_WEIGHT)
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    run_chunk(e, randn(g, L, B, 50, Hq, D), weights=binding.WEIGHTS_SET)
    before, weights = e.dump_state(), e.state_views()["weights"][:, :n].clone()
    for _ in range(75):                                               # (past the ends of two blocks)
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        e.append(kn.unsqueeze(2), vn.unsqueeze(2))
        k, v = torch.cat((k, kn.unsqueeze(3)), 3), torch.cat((v, vn.unsqueeze(3)), 3)
        check_sparse(e, q, k, v, 3)
    after, now = e.dump_state(), e.state_views()["weights"][:, :n + 75]
    assert after["n"] == n + 75 and after["t"] == before["t"] and e.info().evictions == 0
    assert all(np.array_equal(after[x][:, :n], before[x]) for x in ("pos", "ts", "mri"))
    assert np.array_equal(after["pos"][:, n:], np.tile(np.arange(n, n + 75), (L * B * Hkv, 1)))
    assert torch.equal(now[:, :n], weights) and not bool(now[:, n:].any())
    assert e.evict_to(200) == 65                                      # when the caller says so
    assert e.dump_state()["pos"][:, -8:].tolist() == [list(range(n + 67, n + 75))] * (L * B * Hkv)


# ---- a chunk ------------------------------------------------------------------------------------------------------------

def chunk_squares(q, k, v, T, kp=None, vp=None):
    """sum p^2 v^2 of every output."""
    L, B, _, Hq, _ = q.shape
    Hkv, n = k.shape[2:4]
    G, N = Hq // Hkv, 0 if kp is None else kp.shape[3]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):
            for h in range(Hkv):
                kk, vv = k[l, b, h].double(), v[l, b, h].double()
                if N:
                    p = b // (B // kp.shape[1])
                    kk, vv = torch.cat((kp[l, p, h].double(), kk)), torch.cat((vp[l, p, h].double(), vv))
                x = torch.einsum("tgd,jd->tgj", q[l, b, :, h * G:(h + 1) * G].double(), kk) / math.sqrt(D)
                sees = torch.ones(T, N + n, dtype=torch.bool, device="cuda").tril(N + n - T)
                p = torch.softmax(x.masked_fill(~sees[:, None], -math.inf), -1)
                out[l, b, :, h * G:(h + 1) * G] = p.square() @ vv.square()
    return out


def rms_of_tolerance(got, ref, squares, dtype):
    """Weights of the value product are off by at most 2^-8 of themselves, each on its own: the mean square of an output's error is at most
    2^-16 sum p^2 v^2 from them (a third of it for roundings that lie anywhere).  An output's own rounding and the row's sum (2^-13 bounds it) go
    with the output."""
    err = (got.double() - ref).square().mean()
    tol = (2.0 ** -16 * squares + ((TYPES[dtype] + 2.0 ** -13) * ref).square()).mean()
    return float((err / tol).sqrt())


@pytest.mark.parametrize("L,B,Hq,Hkv,context,T", [
    (1, 1, 5, 1, 20000, 1),
    (1, 1, 8, 2, 30001, 4),                         # joined by a launch of its own
    (1, 1, 4, 1, 300000, 1),
    (1, 2, 8, 2, 4000, 200),
    (1, 8, 16, 8, 2100, 300),                       # whole items first
])
def test_chunk_takes_every_key_tile_into_the_value_product(L, B, Hq, Hkv, context, T):
    """Held to the mean square, where no tile of 128 keys can go missing: over long caches one is less than the sum of all roundings'
    largest sizes."""
    g = gen(context + T)
    e, k, v = loaded(g, L, B, Hq, Hkv, context + T)
    q = randn(g, L, B, T, Hq, D)
    got = run_chunk(e, q, torch.float32)
    ref, _, _ = chunk_ref(q, k, v, T)
    squares = chunk_squares(q, k, v, T)
    assert rms_of_tolerance(got, ref, squares, torch.float32) <= 1
    # (the bound sees one tile, wherever it is: an output of all keys but those)
    for at in (0, context // 256 * 128):
        some = v.clone()
        some[..., at:at + 128, :] = 0
        assert rms_of_tolerance(chunk_ref(q, k, some, T)[0], ref, squares, torch.float32) > 1


@pytest.mark.parametrize("Hq,Hkv,B,context,T,N", [
    (16, 8, 8, 2100, 300, 0),                       # 64 units, 3 items each, the last of one row tile
    (28, 4, 20, 1500, 80, 0),                       # 18 tokens of 7 heads, an odd number of tiles
    (8, 8, 12, 300, 700, 1300),                     # behind a prefix
    (32, 8, 2, 9000, 200, 0),                       # an item longer than a block's part
])
def test_chunk_with_whole_items_first(Hq, Hkv, B, context, T, N):
    """Caches that do not stay in L2: a block begins with its whole items and ends with the one that the block before began."""
    g = gen(B + context + T)
    L, n = 1, context + T
    e = engine(L, Hq, Hkv, B, n, weights=True)
    e.set_page_table(np.random.RandomState(n).permutation(e.info().units * e.info().pages_per_unit))
    kp = vp = None
    if N:
        pre, kp, vp = loaded(g, L, 1, Hq, Hkv, N)
        e.attach_prefix(pre)
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, T, Hq, D)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    plan = e.debug_chunk_plan(n, T)
    assert plan["whole_first"] and not plan["whole"] and not plan["joined_apart"]
    for dtype in (torch.float32, torch.bfloat16):
        out = run_chunk(e, q, dtype, weights=binding.WEIGHTS_SET)
        assert torch.equal(out, run_chunk(e, q, dtype, weights=binding.WEIGHTS_SET))
        ref, size, weights = chunk_ref(q, k, v, T, kp, vp)
        assert_chunk(out, ref, size, e.state_views()["weights"][:, :n], weights)
        assert rms_of_tolerance(out, ref, chunk_squares(q, k, v, T, kp, vp), dtype) <= 1
    # a value that only the last token sees, and one in the middle of the chunk
    v[..., n - 1, 5] = math.inf
    v[:, 1::2, :, n - T // 2, 77] = math.nan
    e.reset()
    if N:
        e.attach_prefix(pre)                                          # (a reset detaches it)
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    out = run_chunk(e, q, weights=binding.WEIGHTS_SET)
    ref, size, weights = chunk_ref(q, k, v, T, kp, vp)
    assert_chunk(out, ref, size, e.state_views()["weights"][:, :n], weights)


@pytest.mark.parametrize("tiles", [0, 5])
def test_a_chunk_with_whole_items_first_that_starves_reports_and_recovers(tiles):
    g = gen(36)
    L, B, Hq, Hkv, context, T = 1, 8, 16, 8, 2100, 300
    e, k, v = loaded(g, L, B, Hq, Hkv, context + T, weights=True)
    q = randn(g, L, B, T, Hq, D)
    assert e.debug_chunk_plan(context + T, T)["whole_first"]
    e.set_wait_limit(0.002)
    e.debug_starve_page_ring(tiles)
    e.attend_chunk(q, torch.empty_like(q), weights=binding.WEIGHTS_SET)
    with pytest.raises(binding.LazyEvError) as err:
        e.synchronize()
    assert err.value.code == binding.EDEVICE
    e.debug_starve_page_ring(-1)
    e.set_wait_limit(2.0)
    e.reset()
    e.append(k.transpose(2, 3), v.transpose(2, 3))
    ref, size, w = chunk_ref(q, k, v, T)
    assert_chunk(run_chunk(e, q, weights=binding.WEIGHTS_SET), ref, size, e.state_views()["weights"][:, :context + T], w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("L,B,Hq,Hkv,context,T", [
    (1, 2, 8, 2, 100, 60),                          # whole items, one row tile or two
    (1, 4, 8, 2, 1000, 200),                        # joined by the last block to come
    (1, 1, 8, 2, 9000, 20),                         # by a launch of its own
])
def test_rows_beside_a_later_value_that_is_not_finite(L, B, Hq, Hkv, context, T, dtype):
    """They are computed again and stored over what was there first, by other threads: every time the same."""
    g = gen(context + T)
    n = context + T
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, T, Hq, D)
    v[..., n - 1, 1::8], v[..., n - T // 3, 64::16] = math.inf, math.nan
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k, v=v)
    ref, size, _ = chunk_ref(q, k, v, T)
    out = run_chunk(e, q, dtype)
    assert_chunk(out, ref, size)
    bits = out.view(torch.int32 if dtype == torch.float32 else torch.int16)
    for _ in range(20):
        assert torch.equal(run_chunk(e, q, dtype).view(bits.dtype)[torch.isfinite(out)], bits[torch.isfinite(out)])


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_rows_computed_again_over_a_long_cache_keep_nobody_waiting(value):
    """The last token's value reaches no other row, and the rows that it had got into are done again without a wait that gives up."""
    g = gen(42)
    L, B, Hq, Hkv, n, T = 1, 20, 32, 8, 65536, 64                     # more items than blocks: behind most pieces of work there is another
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, T, Hq, D)
    v[..., n - 1, :] = value
    e, k, v = loaded(g, L, B, Hq, Hkv, n, k=k, v=v)
    e.set_wait_limit(0.01)
    out = run_chunk(e, q)
    assert not bool(torch.isfinite(out[:, :, -1]).any()) and bool(torch.isfinite(out[:, :, :-1]).all())
    for b, h in ((0, 0), (7, 3), (19, 7)):
        at = (slice(None), slice(b, b + 1), slice(None), slice(4 * h, 4 * h + 4))
        ref, size, _ = chunk_ref(q[at], k[:, b:b + 1, h:h + 1], v[:, b:b + 1, h:h + 1], T)
        assert_chunk(out[at], ref, size)


def test_a_chunk_of_more_work_than_a_launch_counts_is_refused():
    g = gen(43)
    L, B, Hq, Hkv, n = 1, 1, 4, 1, 4400000
    e = engine(L, Hq, Hkv, B, n)
    one = randn(g, L, B, 1, Hkv, D)
    e.append(one.expand(L, B, n, Hkv, D), one.expand(L, B, n, Hkv, D))
    assert e.debug_chunk_plan(n, n)["blocks"] == 0 and e.debug_chunk_plan(n, n // 2)["blocks"] > 0
    q, out = (torch.empty(L, B, n, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    e.reserve_chunk(n)
    launches = e.info().launches
    with pytest.raises(binding.LazyEvError) as err:
        e.attend_chunk(q, out)
    assert err.value.code == binding.EINVAL and "not supported" in str(err.value) and e.info().launches == launches
    q, out = randn(g, L, B, 100, Hq, D), out[:, :, :100]
    e.attend_chunk(q, out)
    e.synchronize()
    want = one.double().expand(L, B, 100, Hkv, D).repeat_interleave(Hq, 3)
    assert bool(((out.double() - want).abs() <= (2.0 ** -7 + 2.0 ** -13 + 2.0 ** -16) * want.abs()).all())
    for n, tokens in ((0, 0), (5, 0), (5, 6), (5, -1), (e.info().capacity + 1, 4)):
        with pytest.raises(binding.LazyEvError) as err:
            e.debug_chunk_plan(n, tokens)
        assert err.value.code == binding.EINVAL


# ---- weights of decode steps ----------------------------------------------------------------------------------------------

def joint_probabilities(q, kp, k):
    """Of the own tokens, averaged over a group's heads: q [L, B, Hq, D]; kp [L, P, Hkv, N, D]; k [L, B, Hkv, n, D]."""
    L, B, Hkv, n = k.shape[:4]
    G, N = q.shape[2] // Hkv, kp.shape[3]
    kk = torch.cat((kp.double().repeat_interleave(B // kp.shape[1], 1), k.double()), 3)
    x = torch.einsum("lbhgd,lbhjd->lbhgj", q.double().unflatten(2, (Hkv, G)), kk) / math.sqrt(D)
    return torch.softmax(x, -1)[..., N:].mean(3).flatten(0, 2)


@pytest.mark.parametrize("L,B,Hq,Hkv,n", [
    (2, 6, 28, 4, 333),                             # a block per unit
    (4, 40, 16, 4, 70),                             # a warp per unit
    (4, 40, 16, 4, 0),                              # no own token before the first step
])
@pytest.mark.parametrize("how", ["device", "rows", "host", "async"])
def test_decode_steps_behind_a_prefix_add_their_weights(L, B, Hq, Hkv, n, how):
    g = gen(n + L)
    N = 200
    pre, kp, vp = loaded(g, L, 2, Hq, Hkv, N)
    e = engine(L, Hq, Hkv, B, n + 4, weights=True)
    e.attach_prefix(pre)
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    if n:
        e.prefill(k, v)
    total = torch.zeros(L * B * Hkv, n, device="cuda")
    exact = total.double()
    for _ in range(3):
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        k = torch.cat((k, kn.unsqueeze(3)), 3)
        if how in ("device", "rows"):
            out = torch.empty_like(q)
            (e.decode_step if how == "device" else e.decode_step_rows)(q, kn, vn, out)
        else:
            host = [x.cpu().pin_memory() for x in (q, kn, vn)]
            out = torch.empty(q.shape, dtype=torch.bfloat16).pin_memory()
            if how == "host":
                e.decode_step_host(*host, out)
            else:
                e.decode_step_host_async(*host, out)
                e.host_wait(0)
        e.synchronize()
        n += 1
        views = e.state_views()
        total = torch.cat((total, torch.zeros(total.shape[0], 1, device="cuda")), 1) + views["pbar"][:, :n]
        assert torch.equal(views["weights"][:, :n], total)            # the same float32 sums
        exact = torch.cat((exact, torch.zeros(exact.shape[0], 1, dtype=torch.float64, device="cuda")), 1) + joint_probabilities(q, kp, k)
        assert bool(((views["weights"][:, :n].double() - exact).abs() <= (2.0 ** -13 + 2.0 ** -14) * exact + 1e-30).all())


@pytest.mark.parametrize("how", ["host", "async"])
def test_wide_steps_from_host_buffers_add_their_weights(how):
    """More units than blocks: the step runs in ranges of units."""
    g = gen(37)
    L, B, Hq, Hkv, n = 14, 32, 28, 4, 400
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    engines = [engine(L, Hq, Hkv, B, n + 4, weights=True) for _ in range(2)]
    for e in engines:
        e.prefill(k, v)
    out, ho = torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(L, B, Hq, D, dtype=torch.bfloat16).pin_memory()
    for step in range(3):
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        engines[0].decode_step(q, kn, vn, out)
        host = [x.cpu().pin_memory() for x in (q, kn, vn)]
        if how == "host":
            engines[1].decode_step_host(*host, ho)
        else:
            engines[1].decode_step_host_async(*host, ho)
            engines[1].host_wait(0)
        for e in engines:
            e.synchronize()
        a, b = (e.state_views()["weights"][:, :n + step + 1] for e in engines)
        assert torch.equal(a, b) and torch.equal(out.cpu(), ho) and bool((a.sum(1) - step - 1 <= 1e-4).all())
    assert how == "async" or engines[1].info().host_ranges >= 3       # (of the last host step)


# ---- into another cache ------------------------------------------------------------------------------------------------------

def test_evict_to_between_two_handles_behind_the_same_prefix():
    g = gen(38)
    L, B, P, Hq, Hkv, N, n, keep = 2, 4, 2, 8, 2, 150, 300, 100
    pre, kp, vp = loaded(g, L, P, Hq, Hkv, N)
    big, small = engine(L, Hq, Hkv, B, n, weights=True, n_recent=16, window=16), engine(L, Hq, Hkv, B, keep, weights=True)
    for e in (big, small):
        e.attach_prefix(pre)
        e.set_score_mode(binding.SCORE_WEIGHT)
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, 40, Hq, D)
    big.append(k.transpose(2, 3), v.transpose(2, 3))
    run_chunk(big, q, weights=binding.WEIGHTS_SET)
    before, w = big.dump_state(), big.state_views()["weights"][:, :n].cpu().numpy()
    assert big.evict_to(keep, small) == n - keep
    check_kept(before, None, small, k, v, w, keep, 16, 0)
    assert big.evict_to(keep) == n - keep
    check_kept(before, None, big, k, v, w, keep, 16, 0)
    assert small.info().next_position == big.info().next_position == N + n
    for _ in range(3):                                                # both go on alike, over the prefix and what was kept
        q, kn, vn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
        a, b = torch.empty_like(q), torch.empty_like(q)
        big.decode_step(q, kn, vn, a)
        small.decode_step(q, kn, vn, b)
        x, y = big.dump_state(kv=True, score=True), small.dump_state(kv=True, score=True)
        assert torch.equal(a, b) and all(np.array_equal(x[i], y[i]) for i in ("pos", "ts", "mri", "k", "v", "score"))
    kk, vv = (torch.from_numpy(x[i].view(np.int16).copy()).view(torch.bfloat16).view(L, B, Hkv, -1, D).cuda() for i in ("k", "v"))
    ref, size, _ = chunk_ref(q[:, :, None], kk, vv, 1, kp, vp)
    assert bool(((a.double() - ref[:, :, 0]).abs() <= 2.0 ** -8 * ref[:, :, 0].abs() + 2.0 ** -13 * size[:, :, 0]).all())


def test_a_cut_into_another_handle_is_not_among_the_profiles_evictions():
    g = gen(39)
    e, k, v = loaded(g, 1, 2, 8, 2, 200, weights=True)
    e.set_score_mode(binding.SCORE_WEIGHT)
    e.set_profiling(True)
    assert e.evict_to(100, engine(1, 8, 2, 2, 100)) == 100
    p = e.get_profile()
    assert p.select_launches == 0 and p.select_bytes == 0 and p.compact_launches == 0
    assert e.evict_to(100) == 100
    p = e.get_profile()
    assert p.select_launches == 1 and p.compact_launches == 1


# ---- the binding -----------------------------------------------------------------------------------------------------------------

def test_workspaces_of_growing_chunks_do_not_pile_up():
    e, _, _ = loaded(gen(40), 2, 4, 16, 2, 2000, weights=True)
    largest = 0
    for tokens in range(1, 2001, 13):
        e.reserve_chunk(tokens, binding.WEIGHTS_SET)
        largest = max(largest, e._chunk_room[tokens, binding.WEIGHTS_SET])
        assert e._chunk_space[-1].numel() >= largest
    assert sum(x.numel() for x in e._chunk_space) <= 4 * largest


def test_a_snapshot_whose_weights_do_not_fit_is_refused():
    g = gen(41)
    make = lambda: engine(1, 8, 2, 1, 64, weights=True)
    a, b = make(), make()
    for e in (a, b):
        e.set_score_mode(binding.SCORE_WEIGHT)
    a.prefill(randn(g, 1, 1, 2, 50, D), randn(g, 1, 1, 2, 50, D))
    a.state_views()["weights"][:, :50] = torch.rand(2, 50, generator=g, device="cuda")
    snap = a.dump_state(kv=True, score=True)
    for bad in (snap["score"][:, :49], snap["score"][:1], snap["score"][0, 0]):
        with pytest.raises(ValueError):
            b.load_state(dict(snap, score=bad), 50)
    b.load_state(dict(snap, score=None), 50)                          # (none: zeros)
    assert not bool(b.state_views()["weights"][:, :50].any())
    b.reset()
    b.load_state(snap, 50)
    assert torch.equal(b.state_views()["weights"][:, :50], a.state_views()["weights"][:, :50])
