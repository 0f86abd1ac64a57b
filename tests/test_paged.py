"""The operators of the paged 8-bit cache on the GPU, against the plain model in 64 bits of paged_model.py."""
import itertools
import math
import random

import pytest
import torch

import paged_model as M

pytestmark = pytest.mark.gpu
BT = 64
TYPES = [(torch.float16, "int8"), (torch.float16, "e4m3"), (torch.bfloat16, "int8"), (torch.bfloat16, "e4m3")]
IDS = ["fp16-int8", "fp16-e4m3", "bf16-int8", "bf16-e4m3"]


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2509_00579_amd import binding
    binding.load()
    return binding


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda:0")


class World:
    """A cache with sequences in it: appends go to the GPU and into the model."""

    def __init__(self, gpu, batch, H, G, D, dtype, codes, max_pages, seed=0, garbage=True):
        self.gen = torch.Generator().manual_seed(seed)
        self.batch, self.H, self.Hq, self.D, self.dtype = batch, H, H * G, D, dtype
        n_pages = batch * max_pages + 2
        self.cache = gpu.PagedCache(H, H * G, n_pages, batch + 1, head_dim=D, dtype=dtype, codes=codes)
        if garbage:  # what is not written yet is never looked at
            self.cache.k_tail.fill_(math.nan)
            self.cache.v_tail.fill_(math.nan)
            self.cache.scales.fill_(math.nan)
        self.table = torch.randperm(n_pages, generator=self.gen)[:batch * max_pages].view(batch, max_pages)
        self.tails = torch.randperm(batch + 1, generator=self.gen)[:batch]
        self.d_table, self.d_tails = _i32(self.table), _i32(self.tails)
        self.seqs, self.lens = M.Sequences(batch), [0] * batch
        self.scale_c = torch.exp(0.5 * torch.randn((H, D), generator=self.gen, dtype=torch.float64))
        self.scale_c[:, :2] *= 10

    def rand(self, *shape):
        return torch.randn(shape, generator=self.gen, dtype=torch.float64)

    def tokens(self, n):
        k = (self.rand(n, self.H, self.D) * self.scale_c).to(self.dtype)
        return k, self.rand(n, self.H, self.D).to(self.dtype), self.rand(n, self.Hq, self.D).to(self.dtype)

    def append(self, counts, k, v, q=None, rope=None, positions=None, starts=True, **kw):
        """counts[b] new tokens of every sequence, rows of k, v, q one after the other."""
        n = sum(counts)
        seq = [b for b, c in enumerate(counts) for _ in range(c)]
        place = [self.lens[b] + i for b, c in enumerate(counts) for i in range(c)]
        self.lens = [a + c for a, c in zip(self.lens, counts)]
        args = dict(rope=None, positions=None)
        pos = torch.tensor(place)[None] if positions is None else positions
        if rope is not None:
            cos_sin, inter, sections, binding = rope
            args["rope"] = binding.Rope(cos_sin.cuda(), inter, sections)
            if positions is not None:
                args["positions"] = _i32(positions)
            kr, size = M.rotate(k[:n].double(), cos_sin, pos, inter, sections)
        else:
            kr, size = k[:n].double(), torch.zeros_like(k[:n], dtype=torch.float64)
        for i in range(n):
            self.seqs.add(seq[i], [kr[i]], [size[i]], [v[i].double()])
        if starts:
            args["starts"] = _i32(list(itertools.accumulate([0] + list(counts))))
        got = self.cache.append(k.cuda(), v.cuda(), _i32(self.lens), self.d_table, self.d_tails,
                                q=None if q is None else q.cuda(), **args, **kw)
        if q is not None:
            want, size = M.rotate(q[:n].double(), rope[0], pos, rope[1], rope[2]) if rope else (q[:n].double(), 0 * q[:n].double())
            slack = 3 * 2.0 ** -24 * size
            tol = slack + torch.finfo(self.dtype).eps / 2 * (want.abs() + slack) + (2.0 ** -25 if self.dtype is torch.float16 else 0)
            err = (got[:n].cpu().double() - want).abs()
            assert bool((err <= tol).all()), float((err - tol).max())
        return got

    def check(self):
        torch.cuda.synchronize()
        self.cache.check()
        M.check_stored(self.cache, self.seqs, self.table, self.tails, self.lens)


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
@pytest.mark.parametrize("H,G,D", [(1, 1, 128), (3, 4, 64), (8, 2, 128)])
def test_append_chunks(gpu, dtype, codes, H, G, D):
    """Ragged chunks, empty ones, chunks that end a block exactly, that begin and end inside blocks, that span several."""
    w = World(gpu, 5, H, G, D, dtype, codes, 8, seed=H + D)
    cos_sin = gpu.Rope.table(600, D).cpu()
    for counts in ([1, 64, 0, 63, 130], [62, 1, 0, 1, 200], [0, 70, 5, 64, 2], [1, 0, 59, 128, 1], [130, 129, 128, 127, 0]):
        k, v, q = w.tokens(sum(counts))
        w.append(counts, k, v, q, rope=(cos_sin, False, None, gpu))
        w.check()


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_append_single_tokens(gpu, dtype, codes):
    """One token per sequence, through the ends of two blocks."""
    w = World(gpu, 3, 2, 3, 64, dtype, codes, 4, seed=5)
    cos_sin = gpu.Rope.table(200, 32).cpu()
    k, v, q = w.tokens(100)
    w.append([61, 0, 39], k, v, q, rope=(cos_sin, True, None, gpu))
    for i in range(70):
        k, v, q = w.tokens(3)
        w.append([1, 1, 1], k, v, q, rope=(cos_sin, True, None, gpu), starts=False)
        if i in (0, 1, 2, 3, 24, 25, 63, 64, 69):
            w.check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot,sections", [(128, 128, [16, 24, 24]), (128, 64, [4, 12, 16]), (64, 32, [8, 8]), (64, 64, [32]), (128, 16, [8])])
def test_append_positions_with_axes(gpu, D, rot, sections, interleaved):
    w = World(gpu, 2, 2, 1, D, torch.float16, "int8", 4, seed=rot)
    cos_sin = gpu.Rope.table(5000, rot, base=1e6).cpu()
    for counts in ([70, 3], [1, 128]):
        k, v, q = w.tokens(sum(counts))
        pos = torch.randint(0, 5000, (len(sections), sum(counts)), generator=w.gen)
        pos[0, 0], pos[-1, -1] = 4999, 0
        w.append(counts, k, v, q, rope=(cos_sin, interleaved, sections, gpu), positions=pos)
        w.check()


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_append_does_not_depend_on_the_division_into_calls(gpu, dtype, codes):
    """The same tokens at once, in chunks and one by one leave the same bits."""
    counts, states = [150, 64, 7], []
    cos_sin = gpu.Rope.table(200, 128)
    for way in (0, 1, 2):
        w = World(gpu, 3, 2, 2, 128, dtype, codes, 4, seed=9, garbage=False)
        for t in (w.cache.k_codes, w.cache.v_codes):
            t.view(torch.uint8).zero_()
        for t in (w.cache.scales, w.cache.k_tail, w.cache.v_tail):
            t.zero_()
        k, v, q = (x.cuda() for x in w.tokens(sum(counts)))
        first = [0, 150, 214]
        lens = [0, 0, 0]
        cuts = {0: [[150, 64, 7]], 1: [[1, 63, 7], [100, 1, 0], [49, 0, 0]], 2: [[1, 1, 1]] * 7 + [[1, 1, 0]] * 57 + [[1, 0, 0]] * 86}[way]
        for c in cuts:
            rows = torch.cat([torch.arange(first[b] + lens[b], first[b] + lens[b] + c[b]) for b in range(3)]).cuda()
            lens = [a + x for a, x in zip(lens, c)]
            w.cache.append(k[rows], v[rows], _i32(lens), w.d_table, w.d_tails, rope=gpu.Rope(cos_sin),
                           starts=_i32([0, c[0], c[0] + c[1], sum(c)]))
        assert lens == counts
        n = [x % BT for x in counts]
        tails = [t[int(w.tails[b]), :, :n[b]].clone() for b in range(3) for t in (w.cache.k_tail, w.cache.v_tail)]
        states.append([w.cache.k_codes.view(torch.uint8), w.cache.v_codes.view(torch.uint8), w.cache.scales, *tails])
    for other in states[1:]:
        for a, b in zip(states[0], other):
            assert torch.equal(a, b)


def test_append_strided_rows_in_place_queries_and_rows_behind_the_end(gpu):
    """Slices of a fused projection; queries rotated in place; rows behind the last sequence are left as they were."""
    H, G, D, n = 2, 3, 64, 90
    w = World(gpu, 2, H, G, D, torch.bfloat16, "int8", 4, seed=3)
    cos_sin = gpu.Rope.table(100, 64)
    k, v, q = w.tokens(n + 6)
    fused = torch.cat([x.flatten(1) for x in (q, k, v)], dim=1).cuda()
    dq, dk, dv = (x.unflatten(1, (-1, D)) for x in fused.split([H * G * D, H * D, H * D], dim=1))
    starts = _i32([0, 65, 90])
    want = w.cache.append(k.cuda(), v.cuda(), _i32([65, 25]), w.d_table, w.d_tails, starts=starts, q=q.cuda(), rope=gpu.Rope(cos_sin),
                          q_out=torch.zeros_like(q, device="cuda:0"))
    assert torch.equal(want[90:], torch.zeros_like(want[90:]))
    state = [x.clone() for x in (w.cache.k_codes, w.cache.v_codes, w.cache.scales[w.table[0, 0]], w.cache.k_tail[:, :, :1])]
    page = int(w.table[0, 0])
    for t in (w.cache.k_codes, w.cache.v_codes):
        t[page] = 0
    w.cache.append(dk, dv, _i32([65, 25]), w.d_table, w.d_tails, starts=starts, q=dq, q_out=dq, rope=gpu.Rope(cos_sin))
    now = [w.cache.k_codes, w.cache.v_codes, w.cache.scales[w.table[0, 0]], w.cache.k_tail[:, :, :1]]
    for a, b in zip(state[2:], now[2:]):
        assert torch.equal(a.nan_to_num(7.), b.nan_to_num(7.))
    assert torch.equal(state[0][page], now[0][page]) and torch.equal(state[1][page], now[1][page])
    assert torch.equal(dq[:90], want[:90]) and torch.equal(dq[90:].cpu(), q[90:])
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_append_small_zero_and_large_values(gpu, dtype, codes):
    """Blocks of zeros, of values near the smallest and the largest of the type, of one value among zeros."""
    w = World(gpu, 4, 2, 1, 64, dtype, codes, 2, seed=1)
    k, v, _ = w.tokens(4 * 64)
    big = torch.finfo(dtype).max
    k[:64], v[:64] = 0, 0
    k[64:128] = (k[64:128].double() * (2.0 ** -22 if dtype is torch.float16 else 2.0 ** -126)).to(dtype)
    v[64:128] = (v[64:128].double() * (2.0 ** -22 if dtype is torch.float16 else 2.0 ** -104)).to(dtype)
    k[128:192], v[128:192] = k[128:192].sign() * big, -v[128:192].sign() * big
    k[192:], v[192:] = 0, 0
    k[200, 1, 5], v[255, 0, 63] = -3, 1.5
    w.append([64, 64, 64, 64], k, v)
    w.check()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_append_reports_non_finite_values(gpu, bad):
    """Noticed by the check; NaN in K and 0 in V of that token, a block with such a token has a NaN scale for K; once reported."""
    for which, starts in itertools.product("kv", (True, False)):
        w = World(gpu, 2, 2, 1, 128, torch.float16, "int8", 2, seed=2)
        k, v, _ = w.tokens(64 + 63)
        (k if which == "k" else v)[64 + 3, 1, 40] = bad
        w.append([64, 63], k, v)
        with pytest.raises(gpu.KvcompError) as e:
            w.cache.check()
        assert e.value.status == gpu.ERR_NONFINITE
        w.cache.check()
        t = int(w.tails[1])
        assert torch.isnan(w.cache.k_tail[t, 1, 3]).any() and torch.isfinite(w.cache.k_tail[t, 0, :63]).all()
        assert torch.isfinite(w.cache.v_tail[t, :, :63]).all()
        k, v, _ = w.tokens(2)
        w.append([1, 1], k, v, starts=starts)
        w.cache.check()  # the new tokens are finite
        s = w.cache.scales[int(w.table[1, 0])]
        assert torch.isnan(s[1, 0]) and torch.isfinite(s[0]).all() and torch.isfinite(s[1, 1])
        assert torch.isfinite(w.cache.scales[int(w.table[0, 0])]).all()


def test_append_refuses_on_the_device_what_only_it_sees(gpu):
    """Pages, tails, lengths, starts and positions out of range: nothing is stored for such a sequence, the others are, and the
    check says so once."""
    def fresh():
        w = World(gpu, 3, 2, 1, 64, torch.float16, "int8", 2, seed=4)
        return w, *(x.cuda() for x in w.tokens(3 * 64)[:2])

    rope = gpu.Rope(gpu.Rope.table(64, 64))
    for what in ("page", "page_low", "tail", "length", "length_low", "starts", "starts_end", "more_than_length", "position"):
        w, k, v = fresh()
        lens, table, tails, starts, args = [64, 64, 64], w.table.clone(), w.tails.clone(), [0, 64, 128, 192], {}
        if what == "page":
            table[1, 0] = w.cache.n_pages
        elif what == "page_low":
            table[1, 0] = -1
        elif what == "tail":
            tails[1] = w.cache.n_tails
        elif what == "length":
            lens[1] = 129
        elif what == "length_low":
            lens[1], starts = -5, [0, 64, 64, 128]
        elif what == "starts":
            starts = [0, 64, 60, 124]
        elif what == "starts_end":
            starts, lens = [0, 64, 64, 193], [64, 0, 128]
        elif what == "more_than_length":
            lens[1] = 63
        else:
            pos = torch.arange(192) % 64
            pos[70] = 64
            args = dict(rope=rope, positions=_i32(pos[None]))
        before = [x.clone() for x in (w.cache.scales, w.cache.k_tail, w.cache.v_tail)]
        w.cache.append(k, v, _i32(lens), _i32(table), _i32(tails), starts=_i32(starts), **args)
        with pytest.raises(gpu.KvcompError) as e:
            w.cache.check()
        assert e.value.status == gpu.ERR_STATE, what
        w.cache.check()
        assert torch.isfinite(w.cache.scales[int(w.table[0, 0])]).all(), what
        own = w.cache.scales[int(w.table[2 if what == "starts_end" else 1, 0])]
        assert torch.isnan(own[:, 0]).all(), what  # as it was, or a NaN for the position
        for a, b in zip(before[1:], (w.cache.k_tail, w.cache.v_tail)):
            assert torch.equal(a.nan_to_num(3.), b.nan_to_num(3.)), what


def test_append_single_token_out_of_range(gpu):
    w = World(gpu, 3, 1, 1, 64, torch.float16, "e4m3", 1, seed=8)
    k, v, q = (x.cuda() for x in w.tokens(3))
    out = torch.zeros_like(q)
    w.cache.append(k, v, _i32([65, 0, 1]), w.d_table, w.d_tails, q=q, q_out=out, rope=gpu.Rope(gpu.Rope.table(64, 64)))
    with pytest.raises(gpu.KvcompError) as e:
        w.cache.check()
    assert e.value.status == gpu.ERR_STATE
    assert torch.isnan(out[0]).any() and torch.equal(out[1], torch.zeros_like(out[1])) and torch.equal(out[2], q[2])
    tails = [int(t) for t in w.tails]
    assert torch.isnan(w.cache.k_tail[tails[0]]).all() and torch.isnan(w.cache.k_tail[tails[1]]).all()
    assert torch.equal(w.cache.k_tail[tails[2], :, 0], k[2])


def test_append_captured_and_replayed(gpu):
    """A captured step replays with the lengths of the day: the graph advances them."""
    w = World(gpu, 2, 2, 2, 128, torch.float16, "int8", 3, seed=6)
    k, v, q = w.tokens(62 + 20)
    rope = gpu.Rope(gpu.Rope.table(200, 128))
    w.append([62, 20], k, v, q, rope=(rope.cos_sin.cpu(), False, None, gpu))
    lens, one = _i32(w.lens), _i32([1, 1])
    dk, dv, dq = (torch.empty_like(x[:2], device="cuda:0") for x in (k, v, q))
    out = torch.empty_like(dq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lens.add_(one)
        w.cache.append(dk, dv, lens, w.d_table, w.d_tails, q=dq, q_out=out, rope=rope)
    for _ in range(5):
        k, v, q = w.tokens(2)
        pos = torch.tensor([w.lens])
        w.lens = [x + 1 for x in w.lens]
        kr, size = M.rotate(k.double(), rope.cos_sin.cpu(), pos)
        for b in range(2):
            w.seqs.add(b, [kr[b]], [size[b]], [v[b].double()])
        for a, b in ((dk, k), (dv, v), (dq, q)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want, size = M.rotate(q.double(), rope.cos_sin.cpu(), pos)
        assert bool(((out.cpu().double() - want).abs() <= 3 * 2.0 ** -24 * size + 2.0 ** -11 * want.abs() * 1.001 + 2.0 ** -25).all())
        w.check()


def _close(got, ref, size, spread, plain, dtype):
    """Attention's outputs against 64 bits.  The output is rounded once: eps / 2 of its value (or half the type's smallest step).
    A score is off by what 128 or fewer products summed in binary32 and two or three factors lose, (128 + 8) * 2^-24 of the sum of
    their magnitudes `spread` (bf16 in fp16 parts adds 2^-40 of the largest); numerators and denominator change by that share, and by
    2^-21 for the exponential and the two fp16 parts; sums over the keys in binary32 with a rescaling per tile lose 64 * 2^-24
    more of the weighted magnitudes `size`."""
    got = got.cpu().double()
    eps = torch.finfo(dtype).eps / 2
    share = 2 * 136 * 2.0 ** -24 * spread + 2 * 2.0 ** -21 + 2 * 64 * 2.0 ** -24
    tol = eps * ref.abs() + share * size * (1 + eps) + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -134)
    err = (got - ref).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float((err / tol).max()))


def _reference(w, rows, window, scale, q):
    """Model attention of the last rows[b] tokens of every sequence over what the cache holds; q rows one after the other."""
    parts, at = [[], [], [], []], 0
    now = M.Snapshot(w.cache)
    for b, n in enumerate(rows):
        k, v = now.held(w.table[b], w.tails[b], w.lens[b])
        pos = torch.arange(w.lens[b] - n, w.lens[b])
        for got, x in zip(parts, M.attention(q[at:at + n].double(), k, v, scale, pos, window)):
            got.append(x)
        at += n
    return [torch.cat(x) for x in parts]


def _decode(w, q_len, window=0, scale=None, **kw):
    q = w.rand(w.batch * q_len, w.Hq, w.D).to(w.dtype)
    scale = 1 / math.sqrt(w.D) if scale is None else scale
    got = w.cache.attn_decode(q.cuda(), scale, _i32(w.lens), w.d_table, w.d_tails, q_len=q_len, window=window, **kw)
    torch.cuda.synchronize()
    want64 = _reference(w, [q_len] * w.batch, window, scale, q)
    _close(got, *want64, w.dtype)
    return q, got


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
@pytest.mark.parametrize("H,G,D,q_len", [(1, 1, 128, 1), (2, 8, 128, 1), (3, 3, 64, 1), (2, 4, 64, 5), (1, 7, 128, 4), (2, 16, 128, 1),
                                         (1, 32, 64, 1), (1, 1, 128, 32), (2, 5, 128, 6)])
def test_decode(gpu, dtype, codes, H, G, D, q_len):
    """Lengths from nothing to several blocks, whole and unfinished ones, one row to 32."""
    w = World(gpu, 9, H, G, D, dtype, codes, 12, seed=H * G + D)
    counts = [1, 0, 63, 64, 65, 700, 128, 7, 256]
    k, v, _ = w.tokens(sum(counts))
    w.append(counts, k, v)
    _decode(w, q_len)
    _decode(w, q_len, max_len=700)
    _decode(w, q_len, scale=-0.3)
    w.cache.check()


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 1000, 1 << 30])
def test_decode_sliding_window(gpu, window):
    for dtype, codes, D, q_len in ((torch.float16, "int8", 64, 1), (torch.bfloat16, "e4m3", 128, 3)):
        w = World(gpu, 6, 2, 4, D, dtype, codes, 6, seed=window % 97)
        counts = [1, 64, 65, 200, 383, 0]
        k, v, _ = w.tokens(sum(counts))
        w.append(counts, k, v)
        _decode(w, q_len, window)


@pytest.mark.parametrize("batch,H,G,longest", [(1, 1, 1, 8000), (1, 2, 8, 5000), (3, 8, 2, 3000), (70, 2, 1, 300), (300, 1, 1, 64), (2, 1, 32, 2500)])
def test_decode_split_over_waves_and_workgroups(gpu, batch, H, G, longest):
    """Few long sequences, whose tiles are spread over many workgroups, and many short ones; twice on the same workspace, the
    same bits both times."""
    w = World(gpu, batch, H, G, 64, torch.float16, "int8", longest // 64 + 1, seed=batch)
    rng = random.Random(batch)
    counts = [longest] + [rng.randrange(longest + 1) for _ in range(batch - 1)]
    k, v, _ = w.tokens(sum(counts))
    n = 0
    w.append(counts, k, v)
    q, a = _decode(w, 1)
    b = w.cache.attn_decode(q.cuda(), 1 / 8, _i32(w.lens), w.d_table, w.d_tails)
    assert torch.equal(a, b)
    ws = w.cache.new_workspace()
    c = w.cache.attn_decode(q.cuda(), 1 / 8, _i32(w.lens), w.d_table, w.d_tails, workspace=ws)
    assert torch.equal(a, c) and not ws[:4096].any()


def test_caches_that_share_a_workspace(gpu):
    """Layers on one stream: decode and prefill calls of two caches in turn on one scratch."""
    one = World(gpu, 3, 2, 2, 64, torch.float16, "int8", 30, seed=2)
    two = World(gpu, 2, 1, 8, 64, torch.float16, "e4m3", 40, seed=3)
    two.cache._workspace = one.cache._workspace
    for w, counts in ((one, [1800, 3, 900]), (two, [2400, 70])):
        k, v, _ = w.tokens(sum(counts))
        w.append(counts, k, v)
    for _ in range(2):
        for w in (one, two):
            _decode(w, 1)
            _prefill(w, [3] * w.batch, max_new=3)
    shared = gpu.PagedCache(2, 4, 8, 2, workspace=one.cache.new_workspace())
    assert shared._workspace.numel() >= one.cache._workspace.numel()


def test_decode_strides_and_rows_behind_the_batch(gpu):
    w = World(gpu, 3, 2, 2, 64, torch.bfloat16, "int8", 3, seed=2)
    counts = [70, 64, 10]
    k, v, _ = w.tokens(144)
    w.append(counts, k, v)
    q, want = _decode(w, 2)
    wide = torch.full((8, 4 * 64 + 24), 5.0, dtype=torch.bfloat16, device="cuda:0")
    qs = torch.zeros((6, 3 * 256), dtype=torch.bfloat16, device="cuda:0")
    qs[:, 256:512] = q.cuda().flatten(1)
    got = wide[:6, 8:264].unflatten(1, (4, 64))
    w.cache.attn_decode(qs[:, 256:512].unflatten(1, (4, 64)), 1 / 8, _i32(w.lens), w.d_table, w.d_tails, q_len=2, out=got)
    assert torch.equal(got, want)
    assert (wide[6:] == 5).all() and (wide[:, :8] == 5).all() and (wide[:, 264:] == 5).all()


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_decode_large_and_small_values(gpu, dtype, codes):
    """Scores far apart, a key that takes all the weight, values near the ends of the type's range, queries of zeros."""
    w = World(gpu, 4, 1, 4, 128, dtype, codes, 3, seed=3)
    k, v, _ = w.tokens(4 * 130)
    top = 6e4 if dtype is torch.float16 else 1e30
    k[130:260] = (k[130:260].double() * 30).clamp(-top, top).to(dtype)
    v[130:260] = (v[130:260].double() * (1e4 if dtype is torch.float16 else 1e30)).to(dtype)
    v[260:390] = (v[260:390].double() * (1e-5 if dtype is torch.float16 else 1e-30)).to(dtype)
    k[390:], v[390:] = 0, 0
    w.append([130] * 4, k, v)
    _decode(w, 1)
    _decode(w, 1, scale=0.0)
    q = torch.zeros((4, 4, 128), dtype=dtype, device="cuda:0")
    got = w.cache.attn_decode(q, 1.0, _i32(w.lens), w.d_table, w.d_tails)
    want64 = _reference(w, [1] * 4, 0, 1.0, q.cpu())
    _close(got, *want64, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_decode_non_finite_tokens_reach_only_the_rows_that_see_them(gpu, dtype, codes, D):
    """Inf and NaN in a block and in an unfinished one, hidden by the causal order, by the window or by nothing."""
    w = World(gpu, 3, 2, 1, D, dtype, codes, 3, seed=4)
    k, v, _ = w.tokens(150 + 100 + 70)
    v[3, 1, 5] = math.inf              # sequence 0, block 0, head 1
    k[150 + 98, 0, 7] = math.nan       # sequence 1, unfinished block, head 0: hidden from the rows before
    v[250 + 69, 0, 1] = -math.inf      # sequence 2, its last token
    w.append([150, 100, 70], k, v)
    for window in (0, 50):
        q = w.rand(3 * 3, 2, D).to(dtype)
        got = w.cache.attn_decode(q.cuda(), 0.1, _i32(w.lens), w.d_table, w.d_tails, q_len=3, window=window).cpu()
        nan = torch.isnan(got)
        want = torch.zeros_like(nan)
        want[0:3, 1] = window == 0
        want[4:6, 0] = True   # tokens 98 and 99
        want[8, 0] = True
        assert torch.equal(nan, want), window


def test_decode_places_out_of_range(gpu):
    """A page, a tail or a length that does not fit: NaN for that sequence, the check says so, the others are right."""
    w = World(gpu, 4, 2, 2, 64, torch.float16, "int8", 3, seed=7)
    k, v, _ = w.tokens(4 * 100)
    w.append([100] * 4, k, v)
    q, want = _decode(w, 1)
    for what in ("page", "page_low", "tail", "tail_low", "length", "length_low"):
        lens, table, tails = list(w.lens), w.table.clone(), w.tails.clone()
        if what.startswith("page"):
            table[1, 0] = -1 if what == "page_low" else w.cache.n_pages
        elif what.startswith("tail"):
            tails[1] = -1 if what == "tail_low" else w.cache.n_tails
        else:
            lens[1] = -1 if what == "length_low" else 193
        got = w.cache.attn_decode(q.cuda(), 1 / 8, _i32(lens), _i32(table), _i32(tails))
        assert torch.isnan(got[1]).all() and torch.equal(got[[0, 2, 3]], want[[0, 2, 3]]), what
        with pytest.raises(gpu.KvcompError) as e:
            w.cache.check()
        assert e.value.status == gpu.ERR_STATE
        w.cache.check()
    table = w.table.clone()
    table[:, 2] = 1 << 30  # not needed: the second block is unfinished
    table[:, 1] = -7
    assert torch.equal(w.cache.attn_decode(q.cuda(), 1 / 8, _i32(w.lens), _i32(table), w.d_tails), want)
    w.cache.check()


def test_decode_shared_pages_other_streams_and_replays(gpu):
    """A prefix whose pages two sequences share; two streams with a workspace each; a captured step replayed while eager calls
    run between."""
    w = World(gpu, 2, 4, 4, 128, torch.bfloat16, "e4m3", 40, seed=8)
    k, v, _ = w.tokens(2000)
    k2, v2, _ = w.tokens(30)
    w.append([2000, 0], k, v)
    shared = w.table.clone()
    shared[1, :30] = shared[0, :30]
    for b in range(1920):
        w.seqs.add(1, [w.seqs.k[0][b]], [w.seqs.size[0][b]], [w.seqs.v[0][b]])
    w.table, w.d_table, w.lens[1] = shared, _i32(shared), 1920
    w.append([0, 30], k2, v2)
    q, want = _decode(w, 1)
    lens, dq, out = _i32(w.lens), q.cuda(), torch.empty_like(want)
    side, ws = torch.cuda.Stream(), w.cache.new_workspace()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(10):
        outs.append(w.cache.attn_decode(dq, 1 / math.sqrt(128), lens, w.d_table, w.d_tails))
        with torch.cuda.stream(side):
            outs.append(w.cache.attn_decode(dq, 1 / math.sqrt(128), lens, w.d_table, w.d_tails, workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        w.cache.attn_decode(dq, 1 / math.sqrt(128), lens, w.d_table, w.d_tails, out=out, workspace=ws)
    for shorter in (0, 1, 500, 0):
        lens.copy_(_i32([w.lens[0] // 64 * 64 - 64 * (shorter // 64) if shorter else w.lens[0], w.lens[1]]))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = w.cache.attn_decode(dq, 1 / math.sqrt(128), lens, w.d_table, w.d_tails)
        assert torch.equal(out, eager)
        if not shorter:
            assert torch.equal(out, want)


def _starts(counts):
    return _i32(list(itertools.accumulate([0] + list(counts))))


def _close_chunks(got, ref, size, spread, plain, dtype):
    """As _close, but the weights go into the second product with fp16's 11 bits: each is off by at most 2^-11 of itself, and so
    is the sum that they are divided by, which is taken from the same rounded ones: 2 * 2^-11 of the weighted magnitudes at
    most.  fp16's smallest step is 2^-24, and the reference leaves a row's largest weight at 2^8 at least: half a step is 2^-33 of
    the sum of the weights, for every key that is seen, so 2^-33 of the sum of their magnitudes `plain`.  In the same way the codes
    of a block whose V scale is far below the largest so far are off by half a step of 2^-24 against codes of up to 2^7, at most
    2^-32 of the largest magnitude, under weights whose sum is one; a code is at most 448 / 2^-9 = 2^18 times another of its
    block, and 2^-32 of the largest is within 2^-32 of `plain`.  The first two powers together: 2^-31 of `plain`."""
    got = got.cpu().double()
    eps = torch.finfo(dtype).eps / 2
    share = 2 * 136 * 2.0 ** -24 * spread + 2 * 2.0 ** -11 + 2 * 64 * 2.0 ** -24
    tol = eps * ref.abs() + share * size * (1 + eps) + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -134)
    tol = tol + 2.0 ** -31 * plain.amax(dim=-1, keepdim=True)
    err = (got - ref).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float((err / tol).max()))


def _prefill(w, rows, window=0, scale=None, **kw):
    n = sum(rows)
    q = w.rand(n + 3, w.Hq, w.D).to(w.dtype)
    scale = 1 / math.sqrt(w.D) if scale is None else scale
    out = torch.full(q.shape, 7.0, dtype=w.dtype, device="cuda:0")
    w.cache.attn_prefill(q.cuda(), scale, _starts(rows), _i32(w.lens), w.d_table, w.d_tails, window=window, out=out, **kw)
    torch.cuda.synchronize()
    want64 = _reference(w, rows, window, scale, q)
    _close_chunks(out[:n], *want64, w.dtype)
    assert (out[n:] == 7).all()
    return q, out


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
@pytest.mark.parametrize("H,G,D", [(1, 1, 128), (2, 8, 128), (3, 3, 64), (2, 4, 64), (1, 32, 128), (8, 5, 64)])
def test_prefill(gpu, dtype, codes, H, G, D):
    """Ragged chunks behind pasts of all lengths, chunks of nothing, of one token, of several row tiles."""
    w = World(gpu, 7, H, G, D, dtype, codes, 10, seed=H * G + D)
    first = [0, 64, 63, 1, 130, 0, 100]
    k, v, _ = w.tokens(sum(first))
    w.append(first, k, v)
    rows = [200, 64, 1, 0, 70, 1, 333]
    k, v, _ = w.tokens(sum(rows))
    w.append(rows, k, v)
    _prefill(w, rows, max_new=333, max_len=433)
    _prefill(w, rows)
    _prefill(w, rows, scale=-0.2)
    w.cache.check()


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 1000, 1 << 30])
def test_prefill_sliding_window(gpu, window):
    for dtype, codes, D in ((torch.float16, "int8", 64), (torch.bfloat16, "e4m3", 128)):
        w = World(gpu, 4, 2, 3, D, dtype, codes, 8, seed=window % 91)
        rows = [500, 1, 130, 64]
        k, v, _ = w.tokens(sum(rows))
        w.append(rows, k, v)
        _prefill(w, rows, window)


@pytest.mark.parametrize("batch,H,G,past,new", [(1, 1, 1, 8000, 20), (1, 2, 8, 4000, 3), (2, 1, 4, 3000, 40), (1, 1, 2, 1000, 700), (3, 2, 1, 2000, 1)])
def test_prefill_few_rows_over_a_long_past(gpu, batch, H, G, past, new):
    """The keys are split among workgroups; the same bits twice."""
    for D in (64, 128):
        w = World(gpu, batch, H, G, D, torch.float16, "e4m3", (past + new) // 64 + 1, seed=past)
        counts = [past] + [past // 3] * (batch - 1)
        k, v, _ = w.tokens(sum(counts))
        w.append(counts, k, v)
        k, v, _ = w.tokens(new * batch)
        w.append([new] * batch, k, v)
        q, a = _prefill(w, [new] * batch)
        b = w.cache.attn_prefill(q.cuda(), 1 / math.sqrt(D), _starts([new] * batch), _i32(w.lens), w.d_table, w.d_tails, max_new=new)
        assert torch.equal(a[:new * batch], b[:new * batch])
        _prefill(w, [new] * batch, window=500)


@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_prefill_large_and_small_values(gpu, dtype, codes):
    """Blocks whose V scales lie far apart, growing and falling, scores far apart, zeros."""
    w = World(gpu, 3, 1, 2, 128, dtype, codes, 5, seed=3)
    k, v, _ = w.tokens(3 * 300)
    steps = [1, 1e-3, 30, 1e-2, 300]
    for j, f in enumerate(steps):
        v[64 * j:64 * j + 64] = (v[64 * j:64 * j + 64].double() * f).to(dtype)
        v[600 + 64 * j:664 + 64 * j] = (v[600 + 64 * j:664 + 64 * j].double() * steps[4 - j]).to(dtype)
    k[300:600] = (k[300:600].double() * 30).to(dtype)
    v[364:428], k[428:492] = 0, 0
    w.append([300] * 3, k, v)
    _prefill(w, [300] * 3)
    _prefill(w, [7] * 3)
    _prefill(w, [300] * 3, scale=0.0)


def test_attention_at_the_ends_of_the_range_of_bf16(gpu):
    w = World(gpu, 2, 1, 1, 64, torch.bfloat16, "int8", 3, seed=3)
    k, v, _ = w.tokens(2 * 150)
    v[:150] = (v[:150].sign().double() * 3e38).to(torch.bfloat16)
    v[150:] = (v[150:].double() * 1e-28).to(torch.bfloat16)
    w.append([150, 150], k, v)
    _decode(w, 1)
    _decode(w, 4)
    _prefill(w, [150, 150])
    _prefill(w, [3, 3])
    # keys whose products with the queries binary32 just holds: one of them takes all the weight
    w = World(gpu, 2, 1, 2, 64, torch.bfloat16, "e4m3", 3, seed=3)
    k, v, _ = w.tokens(2 * 150)
    k = (k.double() * 1e34).to(torch.bfloat16)
    w.append([150, 150], k, v)
    q = w.rand(6, 2, 64).to(torch.bfloat16)
    got = w.cache.attn_decode(q.cuda(), 0.125, _i32(w.lens), w.d_table, w.d_tails, q_len=3)
    _close(got, *_reference(w, [3, 3], 0, 0.125, q), w.dtype)
    got = w.cache.attn_prefill(q.cuda(), 0.125, _starts([3, 3]), _i32(w.lens), w.d_table, w.d_tails)
    _close_chunks(got, *_reference(w, [3, 3], 0, 0.125, q), w.dtype)
    # scores around 2^25: an error of theirs is a common factor of a row's weights, or lies within `spread`
    w = World(gpu, 2, 1, 2, 64, torch.bfloat16, "e4m3", 3, seed=3)
    k, v, _ = w.tokens(2 * 150)
    k = (k.double() * 1e5).to(torch.bfloat16)
    w.append([150, 150], k, v)
    _prefill(w, [150, 150])
    w.cache.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,codes", TYPES, ids=IDS)
def test_prefill_non_finite_tokens_reach_only_the_rows_that_see_them(gpu, dtype, codes, D):
    w = World(gpu, 2, 2, 1, D, dtype, codes, 4, seed=4)
    rows = [200, 100]
    k, v, q = w.tokens(300)
    v[70, 1, 5] = math.inf          # sequence 0, block 1, head 1
    k[200 + 98, 0, 7] = math.nan    # sequence 1, unfinished block
    v[200 + 99, 1, 0] = -math.inf
    w.append(rows, k, v)
    for window in (0, 80):
        got = w.cache.attn_prefill(q.cuda(), 0.1, _starts(rows), _i32(w.lens), w.d_table, w.d_tails, window=window).cpu()
        want = torch.zeros(got.shape, dtype=torch.bool)
        want[64:200, 1] = True   # a block's scale stands for all of its tokens
        if window:
            want[127 + window:200, 1] = False
        want[200 + 98:, 0] = True
        want[200 + 99:, 1] = True
        assert torch.equal(torch.isnan(got), want), window


def test_prefill_empty_rows_and_places_out_of_range(gpu):
    """More rows than a length has tokens: zeros for those before the beginning.  Pages, tails, lengths that do not fit: NaN.
    Starts that do not fit: rows left as they were."""
    w = World(gpu, 3, 2, 2, 64, torch.bfloat16, "int8", 3, seed=6)
    k, v, _ = w.tokens(300)
    w.append([100] * 3, k, v)
    rows = [100, 100, 100]
    q, want = _prefill(w, rows)
    more = [110, 100, 3]
    q2 = w.rand(213, 4, 64).to(torch.bfloat16)
    got = w.cache.attn_prefill(q2.cuda(), 1 / 8, _starts(more), _i32(w.lens), w.d_table, w.d_tails)
    want64 = _reference(w, more, 0, 1 / 8, q2)
    _close_chunks(got, *want64, w.dtype)
    assert not got[:10].any()
    got = w.cache.attn_prefill(q2.cuda(), 1 / 8, _starts(more), _i32([0, 100, 100]), w.d_table, w.d_tails)
    assert not got[:110].any()
    w.cache.check()
    for what in ("page", "page_low", "tail", "length", "length_low", "starts", "starts_end", "starts_low"):
        lens, table, tails, starts = list(w.lens), w.table.clone(), w.tails.clone(), [0, 100, 200, 300]
        if what.startswith("page"):
            table[1, 0] = -1 if what == "page_low" else w.cache.n_pages
        elif what == "tail":
            tails[1] = w.cache.n_tails
        elif what.startswith("length"):
            lens[1] = -1 if what == "length_low" else 193
        elif what == "starts":
            starts = [0, 200, 100, 200]
        elif what == "starts_end":
            starts = [0, 100, 200, 304]
        else:
            starts = [-1, 99, 200, 300]
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda:0")
        w.cache.attn_prefill(q.cuda(), 1 / 8, _i32(starts), _i32(lens), _i32(table), _i32(tails), out=out)
        with pytest.raises(gpu.KvcompError) as e:
            w.cache.check()
        assert e.value.status == gpu.ERR_STATE, what
        if what == "starts_end":
            assert torch.equal(out[:200], want[:200]) and (out[200:] == 7).all()
        elif what == "starts_low":
            assert (out[:99] == 7).all() and torch.equal(out[200:300], want[200:300])
        elif not what.startswith("starts"):
            assert torch.isnan(out[100:200]).all(), what
            assert torch.equal(out[:100], want[:100]) and torch.equal(out[200:300], want[200:300]), what


def test_a_prompt_a_chunk_and_steps_as_a_server_runs_them(gpu):
    """Prompt, its attention, single steps that cross a block's end, a drafted step set back, a second chunk: every output against
    the model, the decode steps captured once and replayed with the lengths of the day between eager calls."""
    H, G, D = 2, 4, 128
    w = World(gpu, 3, H, G, D, torch.bfloat16, "e4m3", 8, seed=12)
    cos_sin = gpu.Rope.table(512, D).cpu()
    rope, scale = (cos_sin, False, None, gpu), 1 / math.sqrt(D)

    def chunk(counts):
        k, v, q = w.tokens(sum(counts))
        qr = w.append(counts, k, v, q, rope=rope)
        got = w.cache.attn_prefill(qr, scale, _starts(counts), _i32(w.lens), w.d_table, w.d_tails, max_new=max(counts))
        want64 = _reference(w, counts, 0, scale, qr.cpu())
        _close_chunks(got, *want64, w.dtype)

    chunk([190, 61, 5])
    lens, one = _i32(w.lens), _i32([1, 1, 1])
    dk, dv, dq = (torch.empty((3, n, D), dtype=w.dtype, device="cuda:0") for n in (H, H, H * G))
    qr, out = torch.empty_like(dq), torch.empty_like(dq)
    d_rope, ws = gpu.Rope(cos_sin.cuda()), w.cache.new_workspace()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        lens.add_(one)
        w.cache.append(dk, dv, lens, w.d_table, w.d_tails, q=dq, q_out=qr, rope=d_rope)
        w.cache.attn_decode(qr, scale, lens, w.d_table, w.d_tails, out=out, workspace=ws)
    for step in range(5):
        k, v, q = w.tokens(3)
        pos = torch.tensor([w.lens])
        w.lens = [x + 1 for x in w.lens]
        kr, size = M.rotate(k.double(), cos_sin, pos)
        for b in range(3):
            w.seqs.add(b, [kr[b]], [size[b]], [v[b].double()])
        for a, b in ((dk, k), (dv, v), (dq, q)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want64 = _reference(w, [1] * 3, 0, scale, qr.cpu())
        _close(out, *want64, w.dtype)
        assert torch.equal(out, w.cache.attn_decode(qr, scale, lens, w.d_table, w.d_tails))
    w.check()
    # four drafted tokens, two of them taken back (no block ends among them: 195, 66 and 10 tokens)
    k, v, q = w.tokens(12)
    qr4 = w.append([4, 4, 4], k, v, q, rope=rope)
    got = w.cache.attn_decode(qr4, scale, _i32(w.lens), w.d_table, w.d_tails, q_len=4)
    want64 = _reference(w, [4] * 3, 0, scale, qr4.cpu())
    _close(got, *want64, w.dtype)
    w.lens = [x - 2 for x in w.lens]
    for lists in (w.seqs.k, w.seqs.size, w.seqs.v):
        for x in lists:
            del x[-2:]
    chunk([3, 100, 60])
    w.check()


def test_prefill_captured_on_another_stream_and_replayed_with_other_lengths(gpu):
    """Few rows over long sequences (the keys are split, a second kernel joins them), a padded batch: the launch is fixed when it is
    captured, lengths and starts are read when it runs."""
    w = World(gpu, 3, 2, 4, 128, torch.bfloat16, "int8", 64, seed=31)
    k, v, _ = w.tokens(4000 + 1300)
    w.append([4000, 1300, 0], k, v)
    q = w.rand(40, w.Hq, w.D).to(w.dtype)
    dq, out, scale = q.cuda(), torch.empty((40, w.Hq, 128), dtype=w.dtype, device="cuda:0"), 1 / math.sqrt(128)
    lens, starts = _i32(w.lens), _starts([16, 16, 0])
    side, ws, graph = torch.cuda.Stream(), w.cache.new_workspace(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        w.cache.attn_prefill(dq, scale, starts, lens, w.d_table, w.d_tails, max_new=16, out=out, workspace=ws)
    for rows, back in (([16, 16, 0], (0, 0)), ([1, 0, 0], (0, 0)), ([3, 30, 0], (31, 9)), ([0, 40, 0], (5, 1)), ([16, 16, 0], (0, 0))):
        now = [w.lens[0] - back[0], w.lens[1] - back[1], 0]
        lens.copy_(_i32(now))
        starts.copy_(_starts(rows))
        out.fill_(7.)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        eager = torch.full_like(out, 7.)
        w.cache.attn_prefill(dq, scale, starts, lens, w.d_table, w.d_tails, max_new=16, out=eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        was, w.lens = w.lens, now
        want64 = _reference(w, rows, 0, scale, q)
        w.lens = was
        _close_chunks(out[:sum(rows)], *want64, w.dtype)
        assert (out[sum(rows):] == 7).all()
    w.check()


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_many_rows_of_split_keys(gpu, D):
    """Chunks of 16 sequences whose keys are still worth splitting: the join takes four rows a wave, ragged ends among them."""
    w = World(gpu, 16, 8, 4, D, torch.float16 if D == 64 else torch.bfloat16, "int8", 14, seed=33)
    counts = [(400 + 37 * b) % 830 for b in range(16)]
    k, v, _ = w.tokens(sum(counts))
    w.append(counts, k, v)
    rows = [(10, 16, 0, 1, 3, 33, 9, 15)[b % 8] for b in range(16)]
    k, v, _ = w.tokens(sum(rows))
    w.append(rows, k, v)
    _prefill(w, rows)
    _prefill(w, rows, window=200)
    w.check()


def test_many_sequences_with_empty_places(gpu):
    """More sequences than a wave has lanes, every third place empty, lengths around the ends of blocks."""
    batch = 150
    w = World(gpu, batch, 1, 2, 64, torch.float16, "int8", 3, seed=32)
    counts = [0 if b % 3 == 2 else (1, 63, 64, 65, 127, 128, 129)[b % 7] for b in range(batch)]
    k, v, q = w.tokens(sum(counts))
    w.append(counts, k, v, q)
    got = w.cache.attn_prefill(q.cuda(), 0.125, _starts(counts), _i32(w.lens), w.d_table, w.d_tails)
    _close_chunks(got, *_reference(w, counts, 0, 0.125, q), w.dtype)
    _decode(w, 1)
    _decode(w, 3, window=70)
    w.check()


def test_a_cache_let_go_while_another_stream_uses_it(gpu):
    """Its memory is not handed out again before that stream is through with it."""
    cache = gpu.PagedCache(2, 4, 64, 2, head_dim=64)
    n, at = cache._workspace.numel(), cache._workspace.data_ptr()
    q = torch.zeros((1, 4, 64), dtype=torch.float16, device="cuda:0")
    seqs = (_i32([0]), _i32([[0, 1]]), _i32([0]))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        out = cache.attn_decode(q, 0.1, *seqs)
    del cache
    others = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    busy = not side.query()
    assert not busy or all(x.data_ptr() != at for x in others)
    side.synchronize()
    assert (out == 0).all()


def test_the_binding_refuses(gpu):
    cache = gpu.PagedCache(2, 4, 4, 2, head_dim=64)
    seqs = (_i32([1]), _i32([[0, 1]]), _i32([0]))
    k = torch.zeros((1, 2, 64), dtype=torch.float16, device="cuda:0")
    q = torch.zeros((1, 4, 64), dtype=torch.float16, device="cuda:0")
    for args, kw in (((k, k, *seqs), dict(q_out=q)), ((k, k, *seqs), dict(positions=_i32([[0]]))), ((k.float(), k, *seqs), {}), ((k.cpu(), k, *seqs), {}),
                     ((k, q, *seqs), {}), ((k, k, seqs[0].long(), *seqs[1:]), {}), ((k, k, *seqs), dict(starts=_i32([0]))),
                     ((k, k, seqs[0], seqs[1][0], seqs[2]), {}), ((k[:, :, ::2], k, *seqs), {})):
        with pytest.raises(AssertionError):
            cache.append(*args, **kw)
    with pytest.raises(AssertionError):
        cache.attn_decode(k, 0.1, *seqs)
    with pytest.raises(AssertionError):
        cache.attn_decode(q, 0.1, *seqs, workspace=torch.zeros(8, device="cuda:0"))
    with pytest.raises(gpu.KvcompError):
        cache.attn_decode(q, 0.1, *seqs, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda:0"))
    with pytest.raises(gpu.KvcompError):
        cache.attn_decode(q, 0.1, *seqs, out=q)
    with pytest.raises(gpu.KvcompError):
        cache.attn_prefill(q, math.nan, _i32([0, 1]), *seqs)
    cache.check()


def test_pages_and_tails_far_into_a_large_cache(gpu):
    """Offsets beyond 2^32 bytes and 2^31 elements: the same bits as at the beginning."""
    H, G, D = 8, 2, 128
    gen = torch.Generator().manual_seed(41)
    k, v = (torch.randn((150, H, D), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((150, H * G, D), generator=gen).to(torch.bfloat16).cuda()
    got = []
    for pages, tails, first_page, tail in ((2, 1, 0, 0), (70000, 35000, 69998, 34999)):
        cache = gpu.PagedCache(H, H * G, pages, tails, head_dim=D, dtype=torch.bfloat16)
        seqs = (_i32([150]), _i32([[first_page + 1, first_page, 0]]), _i32([tail]))
        cache.append(k, v, *seqs, starts=_i32([0, 150]))
        chunk = cache.attn_prefill(q, 0.09, _i32([0, 150]), *seqs)
        one = cache.attn_decode(q[-1:], 0.09, *seqs)
        kept = [t[first_page:first_page + 2].view(torch.uint8).clone() for t in (cache.k_codes, cache.v_codes, cache.scales)]
        kept += [t[tail, :, :22].clone() for t in (cache.k_tail, cache.v_tail)]
        cache.check()
        got.append([chunk, one, *kept])
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("G", [16, 32])
def test_decode_the_largest_batch(gpu, G):
    """4096 sequences at once, the most, against 64 at a time: the same bits, one unfinished block each."""
    n, D = 4096, 128
    gen = torch.Generator().manual_seed(42)
    cache = gpu.PagedCache(1, G, 1, n, head_dim=D)
    lens, tails, table = (torch.arange(n) % 7), torch.randperm(n, generator=gen), _i32(torch.zeros((n, 1)))
    starts = _i32(torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]))
    lens, tails = _i32(lens), _i32(tails)
    k, v = (torch.randn((int(starts[-1]), 1, D), generator=gen).half().cuda() for _ in range(2))
    cache.append(k, v, lens, table, tails, starts=starts)
    q = torch.randn((n, G, D), generator=gen).half().cuda()
    got = cache.attn_decode(q, 0.09, lens, table, tails)
    for at in range(0, n, 64):
        part = slice(at, at + 64)
        assert torch.equal(got[part], cache.attn_decode(q[part], 0.09, lens[part], table[part], tails[part])), at
    assert (got[::7] == 0).all() and not (got[1::7] == 0).all()
    cache.check()
