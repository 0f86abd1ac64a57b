"""The paged 8-bit KV cache as cases that can be timed: appending keys and values with the position rotation on the way,
decode attention from the cache, and the attention of prompt chunks.

A page holds 64 tokens of one layer: K codes [pages, H, 64, D], V codes [pages, H, D, 64] (int8 or e4m3) and one fp32 scale
per page, head and tensor [pages, H, 2].  The unfinished block of a sequence stays in 16 bits in a tail [tails, H, 64, D].

A case is a dict of plain values:
  what                       "append", "decode" or "prefill"
  batch, kv_heads, group, head_dim
  dtype, codes               "fp16" or "bf16"; "int8" or "e4m3"
  new                        new tokens of the longest sequence (decode: query rows per sequence)
  past                       tokens of the longest sequence before them
  ragged                     False: all sequences are as long as the longest; True: anything up to that
  window                     tokens that a query sees, itself included (0: all before it)
  rot, interleaved, axes     append only: rotated channels, their order, number of position axes
"""
import math
import random

import torch

own = False

BLOCK = 64
DEVICE = "cuda:0"
LARGEST = {"int8": 127.0, "e4m3": 448.0}
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
TINY = 2.0 ** -100  # a block whose largest value is below this is stored as zeros
BASE = 10000.0


def _case(what, batch, kv_heads, group, new, past, dtype="fp16", codes="int8", head_dim=128, ragged=False, window=0, rot=0,
          interleaved=False, axes=1):
    return dict(what=what, batch=batch, kv_heads=kv_heads, group=group, head_dim=head_dim, dtype=dtype, codes=codes, new=new,
                past=past, ragged=ragged, window=window, rot=rot, interleaved=interleaved, axes=axes)


def listed():
    cases = [
        # One conversation, one token: the smallest append, all launch.
        ("append_1seq_token", _case("append", 1, 8, 4, 1, 1000, rot=128)),
        # A serving batch's step: one token per sequence, a few of them ending a block.
        ("append_64seq_token", _case("append", 64, 8, 8, 1, 1000, "bf16", "e4m3", ragged=True, rot=128)),
        # A long prompt of one sequence, odd length.
        ("append_prompt_16k", _case("append", 1, 8, 4, 16421, 0, rot=128)),
        # Chunks of images and text with positions on three axes, half of a small head rotated, begun and unfinished blocks.
        ("append_12chunks_3axes", _case("append", 12, 8, 2, 1500, 700, "bf16", "e4m3", 64, ragged=True, rot=64, interleaved=True, axes=3)),
        # One head and a short context: the smallest attention, all launch, one tile's latency and the merge.
        ("decode_1head_1k", _case("decode", 1, 1, 1, 1, 999)),
        # One sequence at a long context, as many KV heads as query heads.
        ("decode_32heads_32k", _case("decode", 1, 32, 1, 1, 32767)),
        # A serving batch at long contexts of different lengths, 64 query heads over 8 KV heads.
        ("decode_8x8heads_16k_group8", _case("decode", 8, 8, 8, 1, 16421, "bf16", "e4m3", ragged=True)),
        # Many short conversations, two drafted tokens each, a small head.
        ("decode_64x8heads_1k_draft", _case("decode", 64, 8, 4, 2, 1100, "fp16", "e4m3", 64, ragged=True)),
        # A few tokens per sequence (a short turn, or many drafted tokens): few rows over a long axis.
        ("prefill_4x16_on_4k", _case("prefill", 4, 8, 4, 16, 4001, "bf16", "int8")),
        # A prompt as one chunk.
        ("prefill_8k_prompt", _case("prefill", 1, 8, 4, 8192, 0)),
        # A chunk of a long document behind what is cached.
        ("prefill_512_on_32k_group8", _case("prefill", 1, 8, 8, 512, 32200, "bf16", "e4m3")),
        # A batch of chunks of all lengths, small heads, a sliding window.
        ("prefill_16chunks_window", _case("prefill", 16, 8, 4, 700, 3000, "fp16", "e4m3", 64, ragged=True, window=1024)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))


def draw(rng):
    what = rng.choice(["append", "decode", "decode", "prefill"])
    batch = _log_int(rng, 1, 64)
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16])
    kinds = dict(dtype=rng.choice(["fp16", "bf16"]), codes=rng.choice(["int8", "e4m3"]), head_dim=rng.choice([64, 128, 128]),
                 ragged=rng.random() < 0.7)
    rows = batch * kv_heads * kinds["head_dim"]
    if what == "append":
        longest = max(2, (16384 * 8 * 128) // (rows * (1 + group // 4)))
        new = 1 if rng.random() < 0.4 else _log_int(rng, 2, min(longest, 16384))
        past = _log_int(rng, 1, min(2048, max(2, (1 << 27) // rows))) - 1
        rot = rng.choice([kinds["head_dim"], kinds["head_dim"], kinds["head_dim"] // 2])
        return _case(what, batch, kv_heads, group, new, past, rot=rot, interleaved=rng.random() < 0.3, axes=rng.choice([1, 1, 3]), **kinds)
    if what == "decode":
        new = rng.choice([n for n in (1, 1, 1, 2, 3, 4) if n * group <= 32])
        past = _log_int(rng, 1, min(32768, (1 << 27) // rows)) - 1
        return _case(what, batch, kv_heads, group, new, past, window=rng.choice([0, 0, 0, 1000]), **kinds)
    batch = min(batch, 16)
    rows = batch * kv_heads * kinds["head_dim"]
    past = rng.choice([0, _log_int(rng, 1, min(32768, (1 << 25) // rows))])
    # scores of the longest pairs: no more than those of the longest listed chunks
    most = (1 << 30) // (batch * kv_heads * group)
    new = _log_int(rng, 2, max(2, min(8192, most // max(past, 1), int(math.sqrt(most)))))
    return _case(what, batch, kv_heads, group, new, past, window=rng.choice([0, 0, 0, 500]), **kinds)


def _lengths(case):
    """(new, length with them) of every sequence; the same for every seed."""
    rng = random.Random(11)
    got = []
    for b in range(case["batch"]):
        new, past = case["new"], case["past"]
        if case["ragged"] and b:  # the first sequence is the longest
            past = rng.randrange(past + 1)
            if case["what"] == "append" and case["new"] == 1:
                past |= 0 if rng.random() < 0.9 else 63  # this token ends a block
            elif case["what"] != "decode":
                new = rng.randrange(1, new + 1)
        got.append((new, past + new))
    return got


def _sections(case):
    """Pairs of channels per position axis."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return [pairs]
    first = max(4, pairs // 4 // 4 * 4)
    second = (pairs - first) // 2 // 4 * 4
    return [first, second, pairs - first - second]


def _quantize(x, codes):
    """(codes, scale) of blocks x[..., 64, D], fp32."""
    amax = x.abs().amax(dim=(-1, -2))
    live = amax >= TINY
    safe = torch.where(live, amax, torch.ones_like(amax))
    most = LARGEST[codes]
    scale = torch.where(live, (safe.double() / most).float(), torch.zeros_like(amax))
    inv = torch.where(live, (most / safe.double()).float(), torch.zeros_like(amax))
    y = x * inv[..., None, None]
    return (torch.round(y).to(torch.int8) if codes == "int8" else y.to(torch.float8_e4m3fn)), scale


def _at(pool, index):
    """pool[index] along the first axis, as fp32 (8-bit floats cannot be gathered as they are)."""
    if pool.dtype == torch.float8_e4m3fn:
        return pool.view(torch.uint8)[index].view(torch.float8_e4m3fn).float()
    return pool[index].float()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    H, D, batch, t = case["kv_heads"], case["head_dim"], case["batch"], DTYPES[case["dtype"]]
    heads = H * case["group"]
    new, lens = zip(*_lengths(case))
    need = [-(-n // BLOCK) for n in lens]
    rand = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE)  # noqa: E731
    # pages in any order, as a program that has run for a while has them; entries past a sequence's end stay -1
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE, dtype=torch.int32)
    table = torch.full((batch, max(need) + 1), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    # K with a log-normal scale per channel and four outlier channels per head, V standard normal
    chan = torch.exp(0.5 * rand(H, D))
    chan.scatter_(-1, torch.rand((H, D), generator=gen, device=DEVICE).topk(4, dim=-1).indices, 10.0)
    state = dict(case=case, table=table, scale=1.0 / math.sqrt(D), max_len=max(lens), max_new=max(new))
    if case["what"] == "append" and case["past"] == 0:  # nothing is cached yet
        code = torch.int8 if case["codes"] == "int8" else torch.float8_e4m3fn
        state["k_codes"] = torch.zeros((n_pages, H, BLOCK, D), device=DEVICE).to(code)
        state["v_codes"] = torch.zeros((n_pages, H, D, BLOCK), device=DEVICE).to(code)
        scales = [torch.zeros((n_pages, H), device=DEVICE)] * 2
    else:
        state["k_codes"], ks = _quantize((rand(n_pages, H, BLOCK, D) * chan[:, None]).to(t).float(), case["codes"])
        v, vs = _quantize(rand(n_pages, H, BLOCK, D).to(t).float(), case["codes"])
        state["v_codes"] = v.transpose(-1, -2).contiguous()
        scales = [ks, vs]
    state["scales"] = torch.stack(scales, dim=-1).contiguous()
    state["tails"] = torch.randperm(batch + 1, generator=gen, device=DEVICE, dtype=torch.int32)[:batch]
    state["k_tail"] = (rand(batch + 1, H, BLOCK, D) * chan[:, None]).to(t)
    state["v_tail"] = rand(batch + 1, H, BLOCK, D).to(t)
    tokens = sum(new)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEVICE)  # noqa: E731
    state["lens"] = ints(lens)
    state["starts"] = ints([sum(new[:b]) for b in range(batch + 1)])
    # which sequence a row of new tokens belongs to, and its place among that sequence's new tokens
    state["row_seq"] = torch.repeat_interleave(torch.arange(batch, device=DEVICE), state["starts"].diff().long())
    state["row_place"] = torch.arange(tokens, device=DEVICE) - state["starts"].long()[state["row_seq"]]
    state["q"] = rand(tokens, heads, D).to(t)
    state["out"] = torch.empty_like(state["q"])
    if case["what"] == "append":
        state["k"] = (rand(tokens, H, D) * chan).to(t)
        state["v"] = rand(tokens, H, D).to(t)
        n_pos, pairs = max(lens) + 8, case["rot"] // 2
        angle = torch.arange(n_pos, device=DEVICE, dtype=torch.float64)[:, None] * BASE ** (
            -torch.arange(pairs, device=DEVICE, dtype=torch.float64) / pairs)
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        state["positions"] = None
        if case["axes"] > 1:  # time runs on, height and width are anything in the picture
            time = state["lens"].long()[state["row_seq"]] - state["starts"].long().diff()[state["row_seq"]] + state["row_place"]
            other = torch.randint(0, min(n_pos, 64), (case["axes"] - 1, tokens), generator=gen, device=DEVICE)
            state["positions"] = torch.cat([time[None], other]).int()
        # what these tokens touch of the cache: for every sequence its blocks from the first unfinished one on
        state["first_block"] = (state["lens"] - state["starts"].diff()) // BLOCK
        state["n_blocks"] = max(-(-n // BLOCK) - (n - m) // BLOCK for m, n in zip(new, lens))
    if own:
        from paper_2509_00579_amd import binding
        state["cache"] = binding.PagedCache(H, heads, n_pages, batch + 1, head_dim=D, dtype=t, codes=case["codes"], device=DEVICE,
                                            storage=[state[n] for n in ("k_codes", "v_codes", "scales", "k_tail", "v_tail")])
        if case["what"] == "append":
            state["rope"] = binding.Rope(state["cos_sin"], interleaved=case["interleaved"], sections=_sections(case))
    return state


def _rotate(x, state):
    """x [tokens, heads, D] with its first `rot` channels rotated, fp32."""
    case = state["case"]
    pairs = case["rot"] // 2
    if state["positions"] is None:
        past = state["lens"].long() - state["starts"].long().diff()
        rows = state["cos_sin"][past[state["row_seq"]] + state["row_place"]]
        cos, sin = rows[:, :pairs], rows[:, pairs:]
    else:
        axis = torch.repeat_interleave(torch.arange(case["axes"], device=x.device), torch.tensor(_sections(case), device=x.device))
        pos = state["positions"].long()[axis].t()  # [tokens, pairs]
        cos = state["cos_sin"][:, :pairs].gather(0, pos)
        sin = state["cos_sin"][:, pairs:].gather(0, pos)
    cos, sin = cos[:, None], sin[:, None]
    x = x.float()
    if case["interleaved"]:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., 2 * pairs:]], dim=-1)


def _append(state):
    case, t = state["case"], DTYPES[state["case"]["dtype"]]
    seq, nb, first = state["row_seq"], state["n_blocks"], state["first_block"].long()
    batch, H, D = case["batch"], case["kv_heads"], case["head_dim"]
    lens, tails = state["lens"].long(), state["tails"].long()
    past = lens - state["starts"].long().diff()
    place = past[seq] + state["row_place"] - first[seq] * BLOCK  # from the start of the sequence's first touched block
    block = first[:, None] + torch.arange(nb, device=lens.device)
    ended = ((block + 1) * BLOCK <= lens[:, None])
    page = state["table"].long().gather(1, block.clamp(max=state["table"].shape[1] - 1))
    page = torch.where(ended, page, len(state["k_codes"]))  # blocks that are not written go to a row that is dropped
    begun = lens // BLOCK - first  # the block that stays unfinished, counted like `place`
    for name, x in (("k", _rotate(state["k"], state).to(t)), ("v", state["v"])):
        tail = state[name + "_tail"]
        held = torch.zeros((batch, nb * BLOCK, H, D), dtype=t, device=x.device)
        held[:, :BLOCK] = tail[tails].transpose(1, 2)
        held[seq, place] = x
        held = held.view(batch, nb, BLOCK, H, D).transpose(2, 3)
        codes, scale = _quantize(held.float(), case["codes"])
        if name == "v":
            codes = codes.transpose(-1, -2)
        pool = state[name + "_codes"].view(torch.uint8)
        room = torch.cat([pool, torch.empty_like(pool[:1])])
        room[page.flatten()] = codes.contiguous().view(torch.uint8).flatten(0, 1)
        pool.copy_(room[:-1])
        room = torch.cat([state["scales"], state["scales"][:1]])
        room[page.flatten(), :, 0 if name == "k" else 1] = scale.flatten(0, 1)
        state["scales"].copy_(room[:-1])
        # the unfinished block's new tokens
        slot = lens[seq] // BLOCK == first[seq] + place // BLOCK
        at = torch.where(slot, tails[seq] * BLOCK + place % BLOCK, len(tail) * BLOCK)
        room = torch.cat([tail.transpose(1, 2).flatten(0, 1), torch.empty((1, H, D), dtype=t, device=x.device)])
        room[at] = x
        tail.copy_(room[:-1].view(len(tail), BLOCK, H, D).transpose(1, 2))
    state["out"].copy_(_rotate(state["q"], state).to(t))


def _attend(state, q, pos):
    """q [batch, rows, heads, D] at positions pos [batch, rows]: attention over the cache, fp32."""
    case = state["case"]
    batch, rows, heads, D = q.shape
    H, G = case["kv_heads"], case["group"]
    table, lens = state["table"].long().clamp(min=0), state["lens"].long()
    n_blocks = table.shape[1]
    unfinished = (torch.arange(n_blocks, device=q.device) == (lens // BLOCK)[:, None])[:, :, None, None, None]
    tails = state["tails"].long()
    scales = state["scales"][table][..., None, None]
    k = _at(state["k_codes"], table) * scales[:, :, :, 0]
    k = torch.where(unfinished, state["k_tail"][tails].float()[:, None], k)
    v = _at(state["v_codes"], table).transpose(-1, -2) * scales[:, :, :, 1]
    v = torch.where(unfinished, state["v_tail"][tails].float()[:, None], v)
    k, v = (x.transpose(1, 2).reshape(batch, H, n_blocks * BLOCK, D) for x in (k, v))
    key = torch.arange(n_blocks * BLOCK, device=q.device)
    v = torch.where((key < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    q = q.float().view(batch, rows, H, G, D).permute(0, 2, 3, 1, 4).reshape(batch, H, G * rows, D)
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(batch, H, G, rows, -1) * state["scale"]
    seen = key <= pos[..., None]
    if case["window"]:
        seen &= key > pos[..., None] - case["window"]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p.view(batch, H, G * rows, -1), v) / p.sum(-1).view(batch, H, G * rows, 1)
    return o.view(batch, H, G, rows, D).permute(0, 3, 1, 2, 4).reshape(batch, rows, heads, D)


def run(state):
    case = state["case"]
    if case["what"] == "append":
        if own:
            state["cache"].append(state["k"], state["v"], state["lens"], state["table"], state["tails"],
                                  starts=None if case["new"] == 1 else state["starts"], q=state["q"], q_out=state["out"],
                                  rope=state["rope"], positions=state["positions"])
        else:
            _append(state)
        return {n: state[n] for n in ("k_codes", "v_codes", "scales", "k_tail", "v_tail", "out")}
    if case["what"] == "decode":
        if own:
            return state["cache"].attn_decode(state["q"], state["scale"], state["lens"], state["table"], state["tails"],
                                              q_len=case["new"], window=case["window"], max_len=state["max_len"], out=state["out"])
        pos = state["lens"].long()[:, None] - case["new"] + torch.arange(case["new"], device=DEVICE)
        o = _attend(state, state["q"].view(case["batch"], case["new"], *state["q"].shape[1:]), pos)
        state["out"].copy_(o.flatten(0, 1))
        return state["out"]
    if own:
        return state["cache"].attn_prefill(state["q"], state["scale"], state["starts"], state["lens"], state["table"], state["tails"],
                                           max_new=state["max_new"], max_len=state["max_len"], window=case["window"], out=state["out"])
    new = state["starts"].long().diff()
    place = torch.arange(state["max_new"], device=DEVICE)
    rows = (state["starts"].long()[:-1, None] + place).clamp(max=len(state["q"]) - 1)
    o = _attend(state, state["q"][rows], (state["lens"].long() - new)[:, None] + place)
    state["out"].copy_(o[state["row_seq"], state["row_place"]])
    return state["out"]


def work(case):
    H, G, D = case["kv_heads"], case["group"], case["head_dim"]
    row = H * D  # values of K, or of V, of a token
    bytes_, flops = 0, 0
    for new, length in _lengths(case):
        past = length - new
        if case["what"] == "append":
            ended = length // BLOCK * BLOCK
            bytes_ += new * (2 * row * 2 + 2 * row * G * 2 + case["rot"] * 4)  # K, V, q in and out, cosines and sines
            if ended > past:
                bytes_ += (past % BLOCK) * 2 * row * 2 + (ended - past // BLOCK * BLOCK) * 2 * row
            bytes_ += (length - max(ended, past)) * 2 * row * 2
            flops += new * row * (1 + G) * 3 + new * row * 2
            continue
        first = max(0, past + 1 - case["window"]) if case["window"] else 0
        whole = length // BLOCK * BLOCK
        bytes_ += max(0, whole - first) * 2 * row + (length - max(whole, first)) * 2 * row * 2 + new * row * G * 2 * 2
        if case["window"]:
            seen = sum(min(past + 1 + i, case["window"]) for i in range(new))
        else:
            seen = new * past + new * (new + 1) // 2
        flops += 4 * row * G * seen
    return {"bytes": bytes_, "flops": flops}


# ---- the same in 64 bits, sequence by sequence -------------------------------------------------------------------------

def _to_tail_type(x, t):
    return x.float().to(t).double()  # a value in 64 bits is rounded once to the 16 bits it is kept in


def _exact_rotate(x, pos, case):
    """x [tokens, heads, D] in 64 bits, pos [axes, tokens]; cosines and sines as a program hands them over, in 32 bits."""
    pairs = case["rot"] // 2
    y = x.clone()
    edge = 0
    for axis, width in enumerate(_sections(case)):
        for p in range(edge, edge + width):
            angle = pos[axis].double() * BASE ** (-p / pairs)
            c, s = angle.cos().float().double()[:, None], angle.sin().float().double()[:, None]
            i, j = (2 * p, 2 * p + 1) if case["interleaved"] else (p, p + pairs)
            y[..., i] = x[..., i] * c - x[..., j] * s
            y[..., j] = x[..., j] * c + x[..., i] * s
        edge += width
    return y


def _exact_append(case, seed):
    s = prepare(case, seed)
    t, codes, H = DTYPES[case["dtype"]], case["codes"], case["kv_heads"]
    scales = s["scales"].double()
    got = {n: s[n].double() for n in ("k_codes", "v_codes", "k_tail", "v_tail")}
    out = torch.zeros_like(s["q"], dtype=torch.float64)
    at = 0
    for b, (new, length) in enumerate(_lengths(case)):
        rows = slice(at, at + new)
        at += new
        past, slot = length - new, int(s["tails"][b])
        pos = s["positions"][:, rows] if s["positions"] is not None else torch.arange(past, length, device=DEVICE)[None]
        out[rows] = _exact_rotate(s["q"][rows].double(), pos, case)
        for which, x in enumerate((_to_tail_type(_exact_rotate(s["k"][rows].double(), pos, case), t), s["v"][rows].double())):
            tail = got["kv"[which] + "_tail"]
            begun = past % BLOCK
            x = torch.cat([tail[slot, :, :begun].transpose(0, 1), x])  # [tokens from the first touched block on, H, D]
            n = len(x) // BLOCK
            for j in range(n):
                tile = x[j * BLOCK:(j + 1) * BLOCK].transpose(0, 1)
                page = int(s["table"][b, past // BLOCK + j])
                amax = tile.abs().amax(dim=(1, 2))
                scales[page, :, which] = amax / LARGEST[codes]
                y = tile * (LARGEST[codes] / amax)[:, None, None]
                y = torch.round(y) if codes == "int8" else y.float().to(torch.float8_e4m3fn).double()
                got["kv"[which] + "_codes"][page] = y.transpose(1, 2) if which else y
            rest = x[n * BLOCK:]
            keep = begun if n == 0 else 0  # rows of the tail that were there before
            tail[slot, :, keep:len(rest)] = rest[keep:].transpose(0, 1)
    if codes == "int8":  # whole numbers: there is no distance to them
        got["k_codes"] = got["v_codes"] = None
    return dict(got, scales=scales, out=out)


def exact(case, seed):
    if case["what"] == "append":
        return _exact_append(case, seed)
    s = prepare(case, seed)
    H, G, D = case["kv_heads"], case["group"], case["head_dim"]
    out = torch.zeros_like(s["q"], dtype=torch.float64)
    at = 0
    for b, (new, length) in enumerate(_lengths(case)):
        pages = [int(p) for p in s["table"][b, :length // BLOCK]]
        slot, rest = int(s["tails"][b]), length % BLOCK
        pos = torch.arange(length - new, length, device=DEVICE)[:, None]
        key = torch.arange(length, device=DEVICE)
        hidden = key > pos
        if case["window"]:
            hidden |= key <= pos - case["window"]
        index = torch.tensor(pages, dtype=torch.long, device=DEVICE)
        for h in range(H):
            k = s["k_codes"].view(torch.uint8)[index, h].view(s["k_codes"].dtype).double() * s["scales"][index, h, 0].double()[:, None, None]
            v = s["v_codes"].view(torch.uint8)[index, h].view(s["v_codes"].dtype).double() * s["scales"][index, h, 1].double()[:, None, None]
            k = torch.cat([k.reshape(-1, D), s["k_tail"][slot, h, :rest].double()])
            v = torch.cat([v.transpose(1, 2).reshape(-1, D), s["v_tail"][slot, h, :rest].double()])
            for g in range(G):
                x = s["q"][at:at + new, h * G + g].double() @ k.t() * s["scale"]
                x.masked_fill_(hidden, -math.inf)
                out[at:at + new, h * G + g] = torch.softmax(x, dim=-1) @ v
        at += new
    return out
