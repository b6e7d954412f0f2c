"""Row and prefix calls where they can go wrong between their parts: time-outs in blocks with many short pieces of work, values
that must not vanish between two launches, memory on another stream than its own, calls that are refused.  Tolerances are those of
test_gpu_operators.py."""
import ctypes as C
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2506_15969_b200 import binding
from tests.test_gpu_operators import (D, assert_attend, assert_rows, attend_ref, check_attend, engine, freqs, gen, prefixed,
                                      randn, rows_ref)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("share,Hq,Hkv,N,limits", [
    (32, 64, 8, 100, (0, 1, 2)),           # two row tiles, one key tile: pieces of one turn per stream
    (32, 64, 8, 200, (1, 2, 3, 4)),
    (8, 64, 8, 200, (1, 2, 3, 4)),         # one row tile, two key tiles: pieces of one or two turns
    (8, 64, 8, 300, (1, 2, 5)),
    (40, 64, 8, 100, (1, 2, 3)),           # a pair of row tiles and a single one in turn
])
def test_a_prefix_launch_that_starves_among_short_pieces(share, Hq, Hkv, N, limits):
    """Every block walks several short pieces when its key tiles stop coming: whichever warp gives up first, all of them come to the
    end of their walk within the wait limit, the status word tells, and the handle works again after a reset."""
    g = gen(share * N)
    L, P = 11, 4
    B = P * share
    pre, own, *kv = prefixed(g, L, B, P, Hq, Hkv, N, 5)
    assert L * P * Hkv > 2 * 148           # units of the prefix: more than two pieces per block
    q = randn(g, L, B, Hq, D)
    want = check_attend(own, q, *kv)
    out = torch.empty_like(q)
    for tiles in limits:
        own.set_wait_limit(0.002)
        own.debug_starve_page_ring(tiles)
        own.attend(q, out)
        with pytest.raises(binding.LazyEvError) as err:
            own.synchronize()
        assert err.value.code == binding.EDEVICE
        own.debug_starve_page_ring(-1)
        own.set_wait_limit(2.0)
        own.reset()
        own.attach_prefix(pre)
        own.prefill(kv[2], kv[3])
        own.attend(q, out)
        own.synchronize()
        assert torch.equal(out, want)


def test_many_short_pieces_repeat_exactly():
    """Walks of every kind of piece, back to back: right, and the same bits in every run."""
    for i, (L, P, share, Hq, Hkv, N) in enumerate([(11, 4, 32, 64, 8, 100), (11, 4, 40, 64, 8, 130), (11, 4, 8, 64, 8, 300),
                                                   (9, 3, 20, 56, 8, 500), (28, 2, 16, 28, 4, 2048)]):
        g = gen(40 + i)
        pre, own, *kv = prefixed(g, L, P * share, P, Hq, Hkv, N, 3)
        q = randn(g, L, P * share, Hq, D)
        want = check_attend(own, q, *kv)
        out = torch.empty_like(q)
        for _ in range(50):
            own.attend(q, out)
        own.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("L,B,Hq,Hkv,N,n,splits", [
    (1, 4, 8, 2, 40, 5, 1),                # a block per unit
    (1, 4, 8, 2, 300, 0, 1),
    (1, 4, 8, 2, 3000, 700, 1),
    (1, 4, 8, 2, 3000, 700, 3),            # clusters
    (1, 4, 8, 2, 300, 5, 2),               # a block of the cluster has no own token
    (1, 4, 8, 2, 300, 0, 2),
    (1, 40, 8, 2, 700, 20, 0),
    (16, 40, 12, 2, 70, 65, 0),            # a warp per unit
])
@pytest.mark.parametrize("where", ["prefix", "piece", "second", "own"])
def test_nan_logits_do_not_vanish(L, B, Hq, Hkv, N, n, splits, where):
    """Keys of one KV head that give NaN logits: its heads' outputs and probabilities are NaN, whichever launch joins the parts
    (a part without any finite logit is not an absent one), and the other heads' are as ever."""
    if where == "own":
        n = max(n, 16)
    g = gen(N + n)
    kp, ko = randn(g, L, 1, Hkv, N, D), randn(g, L, B, Hkv, n, D)
    if where == "own":
        ko[:, :, 0, :16] = float("nan")    # all of a warp's tokens
    else:
        first, last = {"prefix": (0, N), "piece": (0, 128), "second": (N // 256 * 128, N // 256 * 128 + 128)}[where]
        kp[:, :, 0, first:last] = float("nan")
    pre, own, kp, vp, ko, vo = prefixed(g, L, B, 1, Hq, Hkv, N, n, kp=kp, ko=ko)
    if splits:
        own.set_splits(splits)
    q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    own.attend(q, out)
    own.synchronize()
    G = Hq // Hkv
    pbar = own.state_views()["pbar"].view(L, B, Hkv, -1)[..., :n]
    assert bool(torch.isnan(out[:, :, :G]).all()) and bool(torch.isnan(pbar[:, :, 0]).all())
    ref, size, ref_pbar = attend_ref(q, kp, vp, ko, vo)
    assert_attend(out[:, :, G:], pbar[:, :, 1:], ref[:, :, G:], size[:, :, G:], ref_pbar[:, :, 1:])


@pytest.mark.parametrize("splits,n", [(1, 40), (2, 40), (1, 600), (3, 600)])
def test_nan_logits_do_not_vanish_without_a_prefix(splits, n):
    g = gen(31)
    L, B, Hq, Hkv = 1, 3, 8, 2
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    k[:, :, 0, 16:32] = float("nan")
    e = engine(L, Hq, Hkv, B, n)
    e.prefill(k, v)
    e.set_splits(splits)
    q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    e.attend(q, out)
    e.synchronize()
    pbar = e.state_views()["pbar"].view(L, B, Hkv, -1)[..., :n]
    assert bool(torch.isnan(out[:, :, :4]).all()) and bool(torch.isnan(pbar[:, :, 0]).all())
    none = k[:, :1, :, :0]
    ref, size, ref_pbar = attend_ref(q, none, none, k, v)
    assert_attend(out[:, :, 4:], pbar[:, :, 1:], ref[:, :, 4:], size[:, :, 4:], ref_pbar[:, :, 1:])


@pytest.mark.parametrize("L,B,n,splits", [(16, 40, 65, 0), (1, 5, 65, 1), (1, 5, 700, 3)])      # enough units for a warp each; blocks; clusters
def test_out_at_any_element(L, B, n, splits):
    """`out` needs no alignment beyond its elements': the launch that stores pairs is not taken for an odd one."""
    g = gen(50 + n)
    Hq, Hkv, N = 12, 2, 70
    pre, own, *kv = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    own.set_splits(splits)
    q, kn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D)
    for at in (0, 1, 2, 3, 8):
        buf = torch.full((q.numel() + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = buf[at:at + q.numel()].view(q.shape)
        own.attend(q, out)
        own.synchronize()
        assert_attend(out, own.state_views()["pbar"][:, :n], *attend_ref(q, *kv))
        assert bool((buf[:at] == 7).all()) and bool((buf[at + q.numel():] == 7).all())
    own.decode_step(q, kn, kn, torch.empty(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(q.shape))
    own.synchronize()
    assert own.info().n == n + 1


def test_misaligned_rows_are_refused():
    """What the kernels load as pairs or 16-byte chunks is refused at an odd element, before anything is queued."""
    g = gen(56)
    L, B, Hq, Hkv, n = 1, 2, 8, 2, 6
    odd = lambda x: torch.cat((x.flatten()[:1], x.flatten()))[1:].view(x.shape)      # noqa: E731
    k, q, kn = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D)
    out = torch.empty_like(q)
    rows_q, rows_out = randn(g, n, L, B, Hq, D), torch.empty(n, L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    e = engine(L, Hq, Hkv, B, n)

    def refused(f, *args):
        with pytest.raises(binding.LazyEvError) as err:
            f(*args)
        assert err.value.code == binding.EINVAL and "aligned" in str(err.value)

    launches = e.info().launches
    refused(e.prefill, odd(k), k)
    refused(e.prefill, k, odd(k))
    for mode in (binding.PROMPT_REPLAY, binding.PROMPT_TILED):
        e.set_prompt_mode(mode)
        refused(e.prefill_observed, rows_q, odd(k), k, rows_out)
        refused(e.prefill_observed, odd(rows_q), k, k, rows_out)
    assert e.info().launches == launches and e.info().n == 0
    e.prefill(k, k)
    launches = e.info().launches
    refused(e.attend, odd(q), out)
    refused(e.decode_step, odd(q), kn, kn, out)
    refused(e.decode_step, q, odd(kn), kn, out)
    refused(e.decode_step, q, kn, odd(kn), out)
    lib = binding.lib()
    assert lib.lazyev_attend(e._h, q.data_ptr(), out.data_ptr() + 1) == binding.EINVAL
    assert e.info().launches == launches and e.info().n == n and e.info().t == 0
    e.decode_step(q, kn, kn, odd(out))
    e.synchronize()


def test_positions_after_a_detach_with_no_own_token():
    """A handle that let its prefix go before it held a token is an empty handle: prompts start at position 0 again, in every form."""
    g = gen(32)
    L, B, Hq, Hkv, N, n = 1, 2, 8, 2, 90, 20
    k, v = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    q, kn = randn(g, L, B, Hq, D), randn(g, L, B, Hkv, D)
    out = torch.empty_like(q)
    whole = engine(L, Hq, Hkv, B, n)
    whole.prefill(k, v)
    whole.decode_step(q, kn, kn, out)
    snap = whole.dump_state(kv=True)
    for load in ("prefill", "observed", "append", "state"):
        pre, own = engine(L, Hq, Hkv, 1, N), engine(L, Hq, Hkv, B, n)
        pre.append(*(randn(g, L, 1, N, Hkv, D) for _ in range(2)))
        own.attach_prefix(pre)
        assert own.info().next_position == N
        own.detach_prefix()
        assert own.info().next_position == 0
        if load == "prefill":
            own.prefill(k, v)
        elif load == "observed":
            own.prefill_observed(randn(g, n, L, B, Hq, D), k, v, torch.empty(n, L, B, Hq, D, dtype=torch.bfloat16, device="cuda"))
        elif load == "append":
            own.append(k.transpose(2, 3), v.transpose(2, 3))
        else:
            own.load_state(snap, n)
        if load != "state":
            own.decode_step(q, kn, kn, out)
        assert np.array_equal(own.dump_state()["pos"], np.tile(np.arange(n + 1), (L * B * Hkv, 1))), load
        assert own.info().next_position == n + 1
    # with own tokens the positions stay
    pre, own, *_ = prefixed(g, L, B, 1, Hq, Hkv, N, 5)
    own.detach_prefix()
    assert own.info().next_position == N + 5


def test_the_workspace_belongs_to_the_engines_stream():
    """Work that is still queued on the current stream may write a block that was just freed there; the prefix's workspace, used on the
    engine's stream, must not be that block."""
    g = gen(33)
    L, B, Hq, Hkv, N, n = 1, 8, 32, 8, 3000, 10
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pre, own, *kv = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    q, out = randn(g, L, B, Hq, D), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    size = C.c_size_t()
    assert binding.lib().lazyev_query_prefix_workspace(own._h, pre._h, C.byref(size)) == binding.OK
    own.detach_prefix()
    torch.cuda.synchronize()
    xs = [torch.zeros(size.value // 4, dtype=torch.float32, device="cuda").fill_(1.0) for _ in range(12)]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for x in xs:
        x.fill_(3.0)                       # partial sums that look present
    keep = xs[1::2]                        # (the free blocks between them are of just that size)
    del x, xs
    own.attach_prefix(pre)
    torch.cuda.synchronize()
    own.attend(q, out)
    own.synchronize()
    assert_attend(out, own.state_views()["pbar"][:, :n], *attend_ref(q, *kv))
    del keep


def test_the_engines_memory_belongs_to_its_stream():
    """Nothing queued on the current stream may still write the pool of an engine that was just made for another stream, and nothing
    there may get the pool of one that was just closed while that stream still reads it."""
    g = gen(34)
    L, B, Hq, Hkv, n = 1, 4, 8, 2, 4000
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, Hq, D)
    out = torch.empty_like(q)
    none = k[:, :1, :, :0]
    want = attend_ref(q, none, none, k, v)
    s = torch.cuda.Stream()
    size = engine(L, Hq, Hkv, B, n, stream=s).kv_pool.numel()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    x = torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    x.fill_(64)
    del x
    e = engine(L, Hq, Hkv, B, n, stream=s)
    e.prefill(k, v)
    torch.cuda.synchronize()
    e.attend(q, out)
    e.synchronize()
    assert_attend(out, e.state_views()["pbar"][:, :n], *want)
    out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    e.attend(q, out)
    del e
    y = torch.full((size,), 64, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert bool(((out.double() - want[0]).abs() <= 2.0 ** -8 * want[0].abs() + 2.0 ** -13 * want[1]).all())
    del y


def test_outputs_whose_dimensions_collide_are_refused():
    g = gen(35)
    e = engine(1, 8, 2, 2, 10)
    lib = binding.lib()
    x = randn(g, 1, 2, 4, 8, D)
    pool = torch.empty(1 << 16, dtype=torch.bfloat16, device="cuda")

    def call(batch, token, head, first=0):
        v = binding._ROWS.pack(x.data_ptr(), binding.BF16, *x.stride()[:4])
        o = binding._ROWS.pack(pool.data_ptr() + 2 * first, binding.BF16, 0, batch, token, head)
        a, b = C.create_string_buffer(v), C.create_string_buffer(o)
        return lib.lazyev_norm_rope(e._h, C.addressof(a), None, 4, None, 0, C.addressof(b), None)

    # (2 sequences, 4 tokens, 8 heads)
    for batch, token, head in ((4096, 128, 128), (4096, 1024, 1024), (128, 256, 256), (1024, 1024, 128), (3968, 1024, 128), (512, 1024, 128),
                               (1024, -1024, 128), (640, 128, 512), (4096, 1016, 128),
                               (4096, 1032, 128)):       # (the last token ends at 4120)
        assert call(batch, token, head, 8192) == binding.EINVAL, (batch, token, head)
        assert "overlap" in lib.lazyev_last_error(e._h).decode()
    for batch, token, head in ((4096, 1024, 128), (128, 2048, 256), (512, 128, 1024), (4128, 1032, 128), (-4096, -1024, 128), (128, 8192, 384),
                               (1152, 256, 2304), (128, 768, 3200)):
        pool.zero_()
        assert call(batch, token, head, 32768) == binding.OK, (batch, token, head)
        e.synchronize()
        assert torch.equal(pool.as_strided(x.shape[1:], (batch, token, head, 1), 32768) if min(batch, token, head) > 0 else
                           pool.as_strided(x.shape[1:], (-batch, -token, head, 1), 32768 + batch + 3 * token).flip(0).flip(1), x[0])


@pytest.mark.parametrize("how", ["detach_prefix", "reset"])
def test_a_prefix_let_go_is_not_kept(how):
    g = gen(36)
    L, B, Hq, Hkv, N, n = 1, 8, 8, 2, 2000, 10
    kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
    k, v, q = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D), randn(g, L, B, Hq, D)
    out = torch.empty_like(q)
    s0, s1 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    pre, own = engine(L, Hq, Hkv, 1, N, stream=s0), engine(L, Hq, Hkv, B, n, stream=s1)
    pre.prefill(kp, vp)
    own.attach_prefix(pre)
    own.prefill(k, v)
    size, there = pre.kv_pool.numel(), weakref.ref(pre)
    with torch.cuda.stream(s1):
        torch.cuda._sleep(200_000_000)
    own.attend(q, out)
    getattr(own, how)()
    del pre
    gc.collect()
    assert there() is None
    with torch.cuda.stream(s0):            # its memory comes back behind what still reads it
        y = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ref, bound, _ = attend_ref(q, kp, vp, k, v)
    assert bool(((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -13 * bound).all())
    del y


@pytest.mark.parametrize("dtype,sizes", [(torch.bfloat16, [1.0, 1e18, 2e18, 1e19, 1e25, 1e38, 3e38]),
                                         (torch.float32, [1e-3, 1e18, 3e18, 1e20, 1e30, 3e37, 1e38])])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_of_rows_whose_squares_overflow(dtype, sizes, interleaved):
    """Finite rows of any size have a norm: the squares of elements from 1.6e18 on, 128 of them, do not fit fp32."""
    g = gen(37)
    H = len(sizes)
    e = engine(1, H, H, 1, 1)
    e.set_rope(freqs(64), interleaved=interleaved)
    w = torch.rand(1, D, generator=g, device="cuda") + 0.5
    e.set_head_norm(w, w, 1e-6)
    unit = torch.rand(1, 1, 40, H, D, generator=g, device="cuda", dtype=torch.float64) * 2 - 1
    x = (unit * torch.tensor(sizes, device="cuda", dtype=torch.float64)[:, None]).to(dtype)
    assert bool(torch.isfinite(x).all())
    for tokens in (1, 40):
        q, k = x[:, :, :tokens], x[:, :, :tokens].flip(3)
        for to in (torch.bfloat16, torch.float32):
            qo, ko = torch.empty(q.shape, dtype=to, device="cuda"), torch.empty(k.shape, dtype=to, device="cuda")
            e.norm_rope(q, k, qo, ko)
            e.synchronize()
            for got, rows in ((qo, q), (ko, k)):
                assert_rows(got, *rows_ref(rows, w, 1e-6, [np.arange(tokens)], freqs(64), interleaved), to)
    # a row with an infinity is NaN there and zero elsewhere in its pairs' formula; its neighbours do not notice
    x[0, 0, 0, 1, 5] = float("inf")
    q, qo = x[:, :, :1], torch.empty(1, 1, 1, H, D, dtype=dtype, device="cuda")
    e.norm_rope(q, None, qo, None)
    e.synchronize()
    assert not bool(torch.isfinite(qo[..., 1, 5]).any())
    rest = [h for h in range(H) if h != 1]
    assert_rows(qo[..., rest, :], *rows_ref(q[..., rest, :], w, 1e-6, [np.arange(1)], freqs(64), interleaved), dtype)


def test_a_host_step_that_is_refused_copies_nothing():
    g = gen(38)
    pre, own, *_ = prefixed(g, 1, 4, 1, 8, 2, 30, 5)
    full = binding.Engine(1, 8, 2, D, 62, 1, 2.0)
    full.set_auto_evict(False)
    full.append(randn(g, 1, 1, 64, 2, D), randn(g, 1, 1, 64, 2, D))
    host = [torch.randn(1, 1, h, D).to(torch.bfloat16).pin_memory() for h in (8, 2, 2, 8)]
    for e, code in ((pre, binding.ESTATE), (full, binding.ECAPACITY)):
        e.synchronize()
        before = e.scratch.clone()
        for step in (e.decode_step_host, e.decode_step_host_async):
            with pytest.raises(binding.LazyEvError) as err:
                step(*host)
            assert err.value.code == code
        e.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(e.scratch, before)


def test_info_of_a_warp_per_unit_launch():
    g = gen(39)
    pre, own, *kv = prefixed(g, 16, 40, 1, 12, 2, 70, 65)
    check_attend(own, randn(g, 16, 40, 12, D), *kv)
    inf = own.info()
    assert inf.splits == 1 and inf.grid > 0 and inf.stages >= 1 and inf.smem_bytes > 100 * 1024 and inf.tail_units == 0


def test_binding_refuses_what_does_not_fit():
    g = gen(40)
    L, B, Hq, Hkv = 1, 2, 8, 2
    e = engine(L, Hq, Hkv, B, 10)
    q, k = randn(g, L, B, 4, Hq, D), randn(g, L, B, 4, Hkv, D)
    e.append(k, k)
    q1, out = q[:, :, 0].contiguous(), torch.empty(L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    twice = torch.empty(2 * L, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    bad = [lambda: e.norm_rope(q.double(), None, q, None), lambda: e.append(k.double(), k.double()), lambda: e.norm_rope(q, None, None, None),
           lambda: e.norm_rope(None, k, None, None), lambda: e.norm_rope(None, None, None, None), lambda: e.append(k, None),
           lambda: e.set_head_norm(torch.ones(L, 2 * D, device="cuda")[:, ::2], None, 1e-6),
           lambda: e.attend(q1.float(), out), lambda: e.attend(q1, out.float()), lambda: e.attend(twice, out), lambda: e.attend(q1, twice),
           lambda: e.attend(twice.view(L, B, 2 * Hq, D)[:, :, ::2], out), lambda: e.decode_step_rows(q[:, :, :1], k[:, :, :1], k[:, :, :1], out.float()),
           lambda: e.decode_step_rows(q[:, :, :1], k[:, :, :1], k[:, :, :1], twice), lambda: e.attend(q1.cpu(), out),
           lambda: e.attend(q1, out.cpu()), lambda: e.decode_step_rows(q[:, :, :1], k[:, :, :1], k[:, :, :1], out[:, :1])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert e.info().n == 4 and e.info().t == 0, i
    e.attend(q[:, :, :1].contiguous(), out)      # one token, its dimension there
    e.synchronize()


def test_the_workspace_fits_whatever_the_prefix_comes_to_hold():
    """The size that is asked for once holds for every length of that prefix."""
    g = gen(41)
    for L, B, Hq, Hkv, cap in ((1, 16, 32, 8, 6000), (1, 4, 8, 1, 3000), (4, 8, 8, 2, 5000)):
        pre, own = engine(L, Hq, Hkv, 1, cap), engine(L, Hq, Hkv, B, 2)
        lib, size, first = binding.lib(), C.c_size_t(), None
        at = 0
        for n in (1, 129, 1000, 2305, 2500, cap):
            k = randn(g, L, 1, n - at, Hkv, D) if n > at else None
            if k is None:
                continue
            pre.append(k, k)
            at = n
            assert lib.lazyev_query_prefix_workspace(own._h, pre._h, C.byref(size)) == binding.OK
            first = first or size.value
            assert size.value == first, (n, size.value, first)


def test_a_workspace_asked_for_early():
    """A workspace of the size that was answered for one token, attached after the prefix has grown: nothing is written behind it."""
    g = gen(42)
    L, B, Hq, Hkv, n, cap = 1, 16, 32, 8, 5, 4608                  # 36 key tiles of 8 units: as many parts as there can be
    pre, own = engine(L, Hq, Hkv, 1, cap), engine(L, Hq, Hkv, B, n)
    ko, vo = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    own.prefill(ko, vo)
    kp, vp = randn(g, L, 1, Hkv, cap, D), randn(g, L, 1, Hkv, cap, D)
    pre.append(kp[..., :1, :].transpose(2, 3), vp[..., :1, :].transpose(2, 3))
    lib, size = binding.lib(), C.c_size_t()
    assert lib.lazyev_query_prefix_workspace(own._h, pre._h, C.byref(size)) == binding.OK
    space = torch.full((size.value + (1 << 20),), 171, dtype=torch.uint8, device="cuda")
    pre.append(kp[..., 1:, :].transpose(2, 3), vp[..., 1:, :].transpose(2, 3))
    need = C.c_size_t()
    assert lib.lazyev_query_prefix_workspace(own._h, pre._h, C.byref(need)) == binding.OK and need.value <= size.value
    assert lib.lazyev_attach_prefix(own._h, pre._h, space.data_ptr()) == binding.OK
    check_attend(own, randn(g, L, B, Hq, D), kp, vp, ko, vo)
    assert bool((space[size.value:] == 171).all())
    own.detach_prefix()
    own.synchronize()


def test_work_behind_a_launch_that_gave_up():
    """A warp-per-unit launch that gives up ends behind the prefix launch: the prefix is let go, emptied and filled anew right behind it."""
    g = gen(57)
    L, B, Hq, Hkv, N, n = 16, 40, 12, 2, 700, 65
    pre, own, kp, vp, ko, vo = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    q = randn(g, L, B, Hq, D)
    out = torch.empty_like(q)
    for pages in (0, 1, 0):
        own.set_wait_limit(1e-4)
        own.debug_starve_page_ring(pages)
        own.attend(q, out)
        own.detach_prefix()
        pre.reset()
        kp, vp = randn(g, L, 1, Hkv, N, D), randn(g, L, 1, Hkv, N, D)
        pre.prefill(kp, vp)
        with pytest.raises(binding.LazyEvError):
            own.synchronize()
        pre.synchronize()
        own.set_wait_limit(2.0)
        own.debug_starve_page_ring(-1)
        own.reset()
        own.attach_prefix(pre)
        own.prefill(ko, vo)
        check_attend(own, q, kp, vp, ko, vo)


@pytest.mark.parametrize("how", ["replaced", "closed"])
def test_norm_weights_outlive_the_work_that_reads_them(how):
    """Weights made on another stream, let go while the engine's stream has yet to read them: their memory is not given away before."""
    g = gen(58)
    L, H = 2, 4
    s = torch.cuda.Stream()
    e = engine(L, H, H, 1, 1, stream=s)
    x = randn(g, L, 1, 50, H, D)
    out = torch.empty_like(x)
    w = torch.rand(L, D, generator=g, device="cuda") + 0.5
    want = rows_ref(x, w, 1e-6, [np.arange(50)], [])
    torch.full((L, D), 9.0, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    e.set_head_norm(w, None, 1e-6)
    e.norm_rope(x, None, out, None)
    if how == "replaced":
        e.set_head_norm(None, None, 0.0)
    else:
        del e
    del w
    others = [torch.full((L, D), 9.0, device="cuda") for _ in range(20)]
    torch.cuda.synchronize()
    assert_rows(out, *want, torch.bfloat16)
    del others


@pytest.mark.parametrize("L,P,share,Hq,Hkv,N,n", [
    (12, 3, 1, 24, 8, 2497, 2),            # one row tile: several pieces of many key tiles per block, of odd and even numbers
    (3, 2, 4, 28, 4, 9001, 5),
    (1, 1, 16, 32, 8, 40000, 30),
    (2, 1, 40, 16, 2, 20000, 3),           # two row tiles and a single one in turn
])
def test_prefix_pages_scattered_over_a_large_pool(L, P, share, Hq, Hkv, N, n):
    """Pages far apart, in random order, in a pool of some GB: loads come in out of order, and every stage of the ring is used only
    when its own load is there.  The same bits in every run, and right."""
    g = gen(N)
    B = P * share
    units = L * P * Hkv
    capacity = max(N + 64, 2 ** 32 // (512 * units))
    pre = binding.Engine(L, Hq, Hkv, D, capacity, 64, 2.0, batch=P)
    inf = pre.info()
    pre.set_page_table(np.random.RandomState(N).permutation(inf.units * inf.pages_per_unit))
    kp, vp = randn(g, L, P, Hkv, N, D), randn(g, L, P, Hkv, N, D)
    pre.prefill(kp, vp)
    own = engine(L, Hq, Hkv, B, n)
    own.attach_prefix(pre)
    ko, vo = randn(g, L, B, Hkv, n, D), randn(g, L, B, Hkv, n, D)
    own.prefill(ko, vo)
    q = randn(g, L, B, Hq, D)
    want = check_attend(own, q, kp, vp, ko, vo)
    out, flush = torch.empty_like(q), torch.empty(2 ** 28, dtype=torch.uint8, device="cuda")
    for i in range(100):
        out.zero_()
        flush.fill_(i)                     # (neither pages nor their translations are near)
        own.attend(q, out)
        assert torch.equal(out, want), i
    own.synchronize()


@pytest.mark.parametrize("splits,n", [(2, 9000), (1, 3000), (8, 9000)])
def test_long_own_caches_behind_a_prefix_launch_that_gives_up(splits, n):
    """The decode launch begins beside a prefix launch of few blocks that only ends by its time-out, and its blocks have more pages to
    stream than their rings hold: all of it ends, the status word tells, and the handle works again."""
    g = gen(59)
    L, B, Hq, Hkv, N = 1, 2, 8, 1, 12800
    pre, own, *kv = prefixed(g, L, B, 1, Hq, Hkv, N, n)
    assert own.info().prefix_blocks == 100
    own.set_splits(splits)
    q = randn(g, L, B, Hq, D)
    want = check_attend(own, q, *kv)
    assert own.info().splits == splits
    out = torch.empty_like(q)
    for limit in (0.002, 0.0005):
        own.set_wait_limit(limit)
        own.debug_starve_page_ring(0)
        own.attend(q, out)
        with pytest.raises(binding.LazyEvError) as err:
            own.synchronize()
        assert err.value.code == binding.EDEVICE
        own.debug_starve_page_ring(-1)
        own.set_wait_limit(2.0)
        own.reset()
        own.attach_prefix(pre)
        own.prefill(kv[2], kv[3])
        own.attend(q, out)
        own.synchronize()
        assert torch.equal(out, want)
