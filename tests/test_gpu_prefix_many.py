"""The group attention of more than 64 sequences, whose plan is a kernel of its own: ragged rows, bad slots, several rows and
slices a sequence, every sequence compared; and rows with other sequences of their group beside them."""
import numpy as np
import pytest

from paper_2606_18967_amd import sdrl
from prefix_ref import Batch
from test_gpu_prefix import own_lengths

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q,n_kv,D,sizes,n", [(8, 2, 128, [8] * 9 + [1, 5], 5), (4, 4, 64, [3] * 30, 2), (32, 4, 64, [65], 1),
                                                (64, 32, 64, [40, 1, 1, 40], 3), (4, 2, 64, [1] * 70, 4), (4, 2, 128, [8] * 37 + [1, 7], 1)])
@pytest.mark.parametrize("prefix", [0, 100, 450])
def test_every_sequence(n_q, n_kv, D, sizes, n, prefix):
    x = Batch(n_q, n_kv, D, sizes, [prefix] * len(sizes), own_lengths(sizes, 90, n), n)
    x.check(x.run())
    x.check(x.run(groups=False))
    x.cache.check()


@pytest.mark.parametrize("n_q,n_kv,D,n", [(8, 2, 128, 5), (28, 4, 64, 3), (64, 32, 64, 4)])
def test_ragged_rows(n_q, n_kv, D, n):
    sizes = [8] * 9 + [1, 5]
    lens = np.random.default_rng(n).integers(0, n + 1, sum(sizes))
    lens[8:16] = 0                                                # a whole group that is not there
    lens[-1] = 0
    x = Batch(n_q, n_kv, D, sizes, [260, 64] + [333] * 9, own_lengths(sizes, 90, 7), n, lens=lens.tolist())
    x.check(x.run())
    x.check(x.run(groups=False))
    x.cache.check()


@pytest.mark.parametrize("n_q,n_kv,D,n", [(32, 2, 64, 20), (16, 1, 128, 33)])
def test_several_slices_a_sequence(n_q, n_kv, D, n):
    sizes = [4] * 16 + [3]
    lens = np.random.default_rng(n).integers(0, n + 1, sum(sizes))
    lens[::5] = n
    x = Batch(n_q, n_kv, D, sizes, [130] * len(sizes), own_lengths(sizes, 150, 2), n, lens=lens.tolist())
    x.check(x.run())
    x.check(x.run(groups=False))
    x.cache.check()


@pytest.mark.parametrize("bad", [-1, 1 << 30])
def test_bad_slots(bad):
    """Sequences without a slot, at a run's start, inside and at its end, are zeros; the others are as before."""
    sizes, n = [8] * 9 + [1, 5], 2
    x = Batch(8, 2, 64, sizes, [400] * len(sizes), own_lengths(sizes, 90, 1), n)
    gone = [0, 11, 23, 72, 77]
    x.slots[gone] = bad
    out = x.run()
    with pytest.raises(sdrl.SDError, match="slot"):
        x.cache.check()
    assert (out[gone] == 0).all()
    x.check(out, seqs=[b for b in range(x.B) if b not in gone])


def test_orders():
    sizes = [6] * 12
    own = own_lengths(sizes, 80, 5)
    for seed in range(2):
        x = Batch(8, 2, 128, sizes, [400] * 12, own, 2, order=np.random.default_rng(seed).permutation(72).tolist())
        x.check(x.run())


def test_the_last_position_and_past_it():
    sizes = [35, 35]
    x = Batch(8, 2, 64, sizes, [256, 256], [10] * 70, 3, max_ctx=268)
    out = x.run()
    with pytest.raises(sdrl.SDError, match="position"):
        x.cache.check()
    assert (out[:, 2] == 0).all()
    x.lens_h = np.full(70, 2)
    y = out.clone()
    y[:, 2] = 7
    x.check(y)


@pytest.mark.parametrize("B", [8, 70])
def test_rows_beside_others_of_their_group(B):
    """A sequence's rows with none, some and all of its group beside it: within two calls' bounds of one another."""
    x = Batch(32, 8, 128, [B], [1000], own_lengths([B], 100, 0), 1)
    whole, slots = x.run(), x.slots
    for ids in ([0], [3, 5], list(range(B // 2)), list(range(B - 1, -1, -1))):
        some = sdrl.prefix_attention(x.cache, x.groups, x.layer, slots[ids].contiguous(), x.q[ids].contiguous())
        for at, b in enumerate(ids):
            tol = x.expected(b)[1]
            assert bool(((some[at].double() - whole[b].double()).abs() <= 2 * tol[0]).all()), (ids, b)
