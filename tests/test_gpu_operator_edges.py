"""Row and prefix calls where they can go wrong between their parts: time-outs in blocks with many short pieces of work, values
that must not vanish between two launches, memory on another stream than its own, calls that are refused.  Tolerances are those of
test_gpu_operators.py."""
import pytest
import torch

from paper_2506_15969_b200 import binding
from tests.test_gpu_operators import D, check_attend, engine, gen, prefixed, randn

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
    L, P = 12, 4
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
    for i, (L, P, share, Hq, Hkv, N) in enumerate([(12, 4, 32, 64, 8, 100), (12, 4, 40, 64, 8, 130), (12, 4, 8, 64, 8, 300),
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
