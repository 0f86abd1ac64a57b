"""The paged cache used on several streams: what one of them flags, writes or lets go is not lost to another."""
import math

import pytest
import torch

import test_paged as P

pytestmark = pytest.mark.gpu
gpu = P.gpu


def test_a_check_names_all_that_was_flagged(gpu):
    """A page out of range and an infinite value: the page's status first, both in the message, both forgotten afterwards."""
    w = P.World(gpu, 2, 1, 1, 64, torch.float16, "int8", 2, seed=1)
    k, v, _ = (x.cuda() for x in w.tokens(128))
    v[70, 0, 3] = math.inf
    table = w.table.clone()
    table[0, 0] = w.cache.n_pages
    w.cache.append(k, v, P._i32([64, 64]), P._i32(table), w.d_tails, starts=P._i32([0, 64, 128]))
    with pytest.raises(gpu.KvcompError) as e:
        w.cache.check()
    assert e.value.status == gpu.ERR_STATE
    assert "a page that was needed is outside the cache" in str(e.value) and "an appended token held Inf or NaN" in str(e.value)
    w.cache.check()


def test_checks_while_another_stream_flags(gpu):
    """Two kinds of faults flagged on another stream at every moment of a check: each is reported by this check or the next."""
    w = P.World(gpu, 1, 1, 1, 64, torch.float16, "int8", 2, seed=1)
    k, v, _ = (x.cuda() for x in w.tokens(1))
    bad = v.clone()
    bad[0, 0, 0] = math.nan
    length, long_, side = P._i32([1]), P._i32([129]), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(300):
        w.cache.append(k, v, long_, w.d_table, w.d_tails)  # a length that does not fit
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(500 * i)
            w.cache.append(k, bad, length, w.d_table, w.d_tails)
        said = ""
        for _ in range(2):
            try:
                w.cache.check()
            except gpu.KvcompError as e:
                said += str(e)
            side.synchronize()
        assert "a length or a start does not fit" in said and "an appended token held Inf or NaN" in said, i
    w.cache.check()


@pytest.mark.parametrize("how", ["new_workspace", "a cache that shares one"])
def test_a_workspace_let_go_while_another_stream_uses_it(gpu, how):
    """Its memory is not handed out again before that stream is through with it."""
    cache = gpu.PagedCache(2, 4, 64, 2, head_dim=64)
    ws = cache.new_workspace()
    n, at = ws.numel(), ws.data_ptr()
    q = torch.zeros((1, 4, 64), dtype=torch.float16, device="cuda:0")
    seqs = (P._i32([0]), P._i32([[0, 1]]), P._i32([0]))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        if how == "new_workspace":
            out = cache.attn_prefill(q, 0.1, P._i32([0, 1]), *seqs, workspace=ws)
        else:
            cache = gpu.PagedCache(2, 4, 64, 2, head_dim=64, storage=[cache.k_codes, cache.v_codes, cache.scales, cache.k_tail,
                                                                      cache.v_tail], workspace=ws)
            torch.cuda._sleep(200_000_000)  # making a cache waits for the stream
            out = cache.attn_decode(q, 0.1, *seqs)
            cache._workspace = None
    del ws
    others = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    busy = not side.query()
    assert not busy or all(x.data_ptr() != at for x in others)
    side.synchronize()
    assert (out == 0).all()
