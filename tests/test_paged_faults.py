"""What an append to the paged cache leaves behind where the device finds that a sequence does not fit."""
import pytest
import torch

import test_paged as P

pytestmark = pytest.mark.gpu
gpu = P.gpu


@pytest.mark.parametrize("dtype,codes", P.TYPES, ids=P.IDS)
@pytest.mark.parametrize("which", [0, 1, 2, 70])
def test_an_append_without_a_page_can_be_repeated(gpu, dtype, codes, which):
    """A page out of range, that of the block that the tail has begun, of a later one, of one behind the 64th: the tail keeps its rows, and the
    same call with the right table leaves what it would have left at once."""
    w = P.World(gpu, 2, 2, 1, 64, dtype, codes, 80, seed=which)
    k, v, _ = w.tokens(20 + 50)
    w.append([20, 50], k, v)
    counts = [75 * 64 if which == 70 else 200, 100]
    k, v, _ = (x.cuda() for x in w.tokens(sum(counts)))
    table = w.table.clone()
    table[0, which] = -1 if which else w.cache.n_pages
    before = [t[int(w.tails[0])].clone() for t in (w.cache.k_tail, w.cache.v_tail)]
    starts, lens = P._starts(counts), P._i32([20 + counts[0], 150])
    w.cache.append(k, v, lens, P._i32(table), w.d_tails, starts=starts)
    with pytest.raises(gpu.KvcompError) as e:
        w.cache.check()
    assert e.value.status == gpu.ERR_STATE
    for a, t in zip(before, (w.cache.k_tail, w.cache.v_tail)):
        assert torch.equal(a.nan_to_num(3.0), t[int(w.tails[0])].nan_to_num(3.0))
    w.append([counts[0], 0], k[:counts[0]].cpu(), v[:counts[0]].cpu())  # the other sequence has its tokens
    w.lens[1] += 100
    zero = torch.zeros((2, 64), dtype=torch.float64)
    for i in range(counts[0], sum(counts)):
        w.seqs.add(1, [k[i].cpu().double()], [zero], [v[i].cpu().double()])
    w.check()


def test_a_single_token_without_a_page_can_be_repeated(gpu):
    """The token that ends a block."""
    w = P.World(gpu, 2, 2, 1, 128, torch.float16, "int8", 2, seed=3)
    k, v, _ = w.tokens(63 + 10)
    w.append([63, 10], k, v)
    k, v, _ = w.tokens(2)
    table = w.table.clone()
    table[0, 0] = -5
    w.cache.append(k.cuda(), v.cuda(), P._i32([64, 11]), P._i32(table), w.d_tails)
    with pytest.raises(gpu.KvcompError):
        w.cache.check()
    w.append([1, 1], k, v, starts=False)  # the same once more, the second sequence's too
    w.check()
