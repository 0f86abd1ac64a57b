"""What the paged cache's entry points refuse on the host, before anything reaches a device (no GPU needed: the pointers are
never used)."""
import ctypes as C

import pytest

ALIGNED = 1 << 20


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_kv_heads", "n_q_heads", "head_dim", "data_type", "code_type", "n_pages", "n_tails",
                                         "max_pages")]


class Tensors(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_k_codes", "d_v_codes", "d_scales", "d_k_tail", "d_v_tail", "d_fault")]


class Batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("d_lens", C.c_void_p), ("d_table", C.c_void_p), ("d_tails", C.c_void_p)]


class New(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("d_starts", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("k_stride", C.c_size_t), ("v_stride", C.c_size_t), ("d_q", C.c_void_p), ("d_q_out", C.c_void_p),
                ("q_stride", C.c_size_t), ("q_out_stride", C.c_size_t), ("d_cos_sin", C.c_void_p), ("n_positions", C.c_int32),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32), ("sections", C.c_int32 * 3),
                ("d_positions", C.c_void_p)]


@pytest.fixture(scope="module")
def B():
    from paper_2509_00579_amd import binding, build
    if not build.LIB.exists():
        build.build()
    binding.load()
    return binding


def _config(B, **kw):
    d = dict(n_kv_heads=8, n_q_heads=32, head_dim=128, data_type=0, code_type=0, n_pages=100, n_tails=4, max_pages=16)
    d.update(kw)
    return C.byref(Config(**d))


def _memory(B, **kw):
    d = dict.fromkeys(("d_k_codes", "d_v_codes", "d_scales", "d_k_tail", "d_v_tail", "d_fault"), ALIGNED)
    d.update(kw)
    return C.byref(Tensors(**d))


def _batch(B, **kw):
    d = dict(batch=3, d_lens=ALIGNED, d_table=ALIGNED, d_tails=ALIGNED)
    d.update(kw)
    return C.byref(Batch(**d))


def _new(B, **kw):
    d = dict(n_tokens=10, d_starts=ALIGNED, d_k=ALIGNED, d_v=ALIGNED, k_stride=1024, v_stride=1024, d_q=0, d_q_out=0, q_stride=0,
             q_out_stride=0, d_cos_sin=0, n_positions=0, rot_dim=0, interleaved=0, n_axes=1, sections=(C.c_int32 * 3)(), d_positions=0)
    d.update(kw)
    d["sections"] = (C.c_int32 * 3)(*d["sections"])
    return C.byref(New(**d))


BAD_CONFIGS = [dict(n_kv_heads=0), dict(n_q_heads=33), dict(n_q_heads=0), dict(n_kv_heads=1, n_q_heads=33), dict(head_dim=96),
               dict(data_type=2), dict(data_type=-1), dict(code_type=2), dict(n_pages=0), dict(n_tails=0), dict(max_pages=0),
               dict(max_pages=(1 << 20) + 1)]
BAD_MEMORY = [dict(d_k_codes=0), dict(d_v_codes=0), dict(d_scales=0), dict(d_k_tail=0), dict(d_v_tail=0), dict(d_fault=0),
              dict(d_k_codes=ALIGNED + 8), dict(d_v_codes=ALIGNED + 4), dict(d_k_tail=ALIGNED + 2), dict(d_scales=ALIGNED + 4),
              dict(d_fault=ALIGNED + 1)]
BAD_BATCHES = [dict(batch=-1), dict(d_lens=0), dict(d_table=0), dict(d_tails=0), dict(batch=1 << 20)]


def _refused(B, status):
    assert status == B.ERR_INVALID_ARG
    assert B.load().kvcomp_last_error()


@pytest.mark.parametrize("i", range(len(BAD_CONFIGS) + len(BAD_MEMORY) + len(BAD_BATCHES)))
def test_append_refuses_bad_caches(B, i):
    bad = (BAD_CONFIGS + BAD_MEMORY + BAD_BATCHES)[i]
    cfg, mem, seqs = _config(B), _memory(B), _batch(B)
    if i < len(BAD_CONFIGS):
        cfg = _config(B, **bad)
    elif i < len(BAD_CONFIGS) + len(BAD_MEMORY):
        mem = _memory(B, **bad)
    else:
        seqs = _batch(B, **bad)
    _refused(B, B.load().kvcomp_paged_append(cfg, mem, seqs, _new(B), None))


ROPE = dict(d_cos_sin=ALIGNED, n_positions=100, rot_dim=64, sections=(32,))
Q = dict(d_q=ALIGNED, d_q_out=ALIGNED, q_stride=4096, q_out_stride=4096)


@pytest.mark.parametrize("bad", [
    dict(n_tokens=-1), dict(d_starts=0), dict(n_tokens=1 << 26), dict(d_k=0), dict(d_v=0), dict(d_k=ALIGNED + 8), dict(d_v=ALIGNED + 2),
    dict(k_stride=1023), dict(k_stride=1016), dict(v_stride=1028), dict(Q, d_q=0), dict(Q, d_q_out=0), dict(Q, q_stride=4088),
    dict(Q, q_stride=4100), dict(Q, d_q=ALIGNED + 8), dict(Q, q_out_stride=8192), dict(ROPE, rot_dim=24), dict(ROPE, rot_dim=8),
    dict(ROPE, rot_dim=144, sections=(72,)), dict(ROPE, n_positions=0), dict(ROPE, d_cos_sin=ALIGNED + 4), dict(ROPE, sections=(28,)),
    dict(ROPE, n_axes=0), dict(ROPE, n_axes=4), dict(ROPE, n_axes=2, sections=(16, 16)),
    dict(ROPE, n_axes=2, sections=(14, 18), d_positions=ALIGNED), dict(ROPE, n_axes=3, sections=(36, -8, 4), d_positions=ALIGNED)])
def test_append_refuses_bad_tokens(B, bad):
    _refused(B, B.load().kvcomp_paged_append(_config(B), _memory(B), _batch(B), _new(B, **bad), None))


def test_nothing_to_append_is_fine(B):
    lib = B.load()
    assert lib.kvcomp_paged_append(_config(B), _memory(B), _batch(B), _new(B, n_tokens=0, d_k=0, d_v=0), None) == B.OK
    assert lib.kvcomp_paged_append(_config(B), _memory(B), _batch(B, batch=0, d_lens=0), _new(B, n_tokens=0, d_starts=0), None) == B.OK


def test_null_structures(B):
    lib = B.load()
    good = [_config(B), _memory(B), _batch(B), _new(B)]
    for i in range(4):
        args = list(good)
        args[i] = None
        _refused(B, lib.kvcomp_paged_append(*args, None))
    _refused(B, lib.kvcomp_paged_check(None, None))
    _refused(B, lib.kvcomp_paged_check(_memory(B, d_fault=0), None))


def _decode_args(B, **kw):
    lib = B.load()
    ws = lib.kvcomp_paged_workspace_bytes(_config(B))
    d = dict(q=ALIGNED, q_stride=4096, q_len=1, scale=0.1, window=0, max_len=0, out=2 * ALIGNED, out_stride=4096, ws=ALIGNED, ws_bytes=ws)
    d.update(kw)
    return [*d.values(), None]


def _prefill_args(B, **kw):
    lib = B.load()
    ws = lib.kvcomp_paged_workspace_bytes(_config(B))
    d = dict(q=ALIGNED, q_stride=4096, starts=ALIGNED, n_tokens=50, scale=0.1, window=0, max_new=0, max_len=0, out=2 * ALIGNED,
             out_stride=4096, ws=ALIGNED, ws_bytes=ws)
    d.update(kw)
    return [*d.values(), None]


def test_workspace_size(B):
    lib = B.load()
    assert lib.kvcomp_paged_workspace_bytes(_config(B)) > lib.kvcomp_paged_workspace_bytes(_config(B, head_dim=64)) > 0
    assert lib.kvcomp_paged_workspace_bytes(_config(B, head_dim=80)) == 0 and lib.kvcomp_paged_workspace_bytes(None) == 0


@pytest.mark.parametrize("i", range(len(BAD_CONFIGS) + len(BAD_MEMORY) + len(BAD_BATCHES)))
def test_attention_refuses_bad_caches(B, i):
    bad = (BAD_CONFIGS + BAD_MEMORY + BAD_BATCHES)[i]
    cfg, mem, seqs = _config(B), _memory(B), _batch(B)
    if i < len(BAD_CONFIGS):
        cfg = _config(B, **bad)
    elif i < len(BAD_CONFIGS) + len(BAD_MEMORY):
        mem = _memory(B, **bad)
    else:
        seqs = _batch(B, **bad)
    _refused(B, B.load().kvcomp_paged_attn_decode(cfg, mem, seqs, *_decode_args(B)))
    _refused(B, B.load().kvcomp_paged_attn_prefill(cfg, mem, seqs, *_prefill_args(B)))


COMMON = [dict(q=0), dict(q=ALIGNED + 8), dict(q_stride=4088), dict(q_stride=4100), dict(out=0), dict(out=ALIGNED + 2), dict(out_stride=4000),
          dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=3e38), dict(window=-1), dict(max_len=-1), dict(ws=0), dict(ws=ALIGNED + 8)]


@pytest.mark.parametrize("bad", COMMON + [dict(q_len=0), dict(q_len=-1), dict(q_len=9), dict(q_len=1 << 30)])
def test_decode_refuses_bad_arguments(B, bad):
    _refused(B, B.load().kvcomp_paged_attn_decode(_config(B), _memory(B), _batch(B), *_decode_args(B, **bad)))


@pytest.mark.parametrize("bad", COMMON + [dict(starts=0), dict(starts=ALIGNED + 2), dict(n_tokens=-1), dict(n_tokens=1 << 26), dict(max_new=-1)])
def test_prefill_refuses_bad_arguments(B, bad):
    _refused(B, B.load().kvcomp_paged_attn_prefill(_config(B), _memory(B), _batch(B), *_prefill_args(B, **bad)))


@pytest.mark.parametrize("q,q_stride,out,out_stride,rows", [
    (0, 4096, 0, 4096, 3), (0, 4096, 4080, 4096, 3), (0, 4096, 2 * 4096 + 4088, 4096, 3), (4088, 4096, 0, 4096, 1), (0, 8192, 4088, 8192, 3),
    (0, 12288, 8200, 12288, 3), (12288 + 4088, 12288, 0, 12288, 3), (0, 4096, 4096, 8192, 3), (8, 12288, 0, 4096, 3)])
def test_attention_refuses_outputs_over_queries(B, q, q_stride, out, out_stride, rows):
    kw = dict(q=ALIGNED + 2 * q, out=ALIGNED + 2 * out, q_stride=q_stride, out_stride=out_stride)
    seqs = _batch(B, batch=rows)
    _refused(B, B.load().kvcomp_paged_attn_decode(_config(B), _memory(B), seqs, *_decode_args(B, **kw)))
    _refused(B, B.load().kvcomp_paged_attn_prefill(_config(B), _memory(B), seqs, *_prefill_args(B, n_tokens=rows, **kw)))


@pytest.mark.parametrize("q,q_stride,out,out_stride", [(0, 4096, 3 * 4096, 4096), (0, 12288, 4096, 12288), (8192, 12288, 0, 12288),
                                                       (0, 12288, 2 * 12288 + 4096, 4096), (3 * 12288 + 4096, 12288, 0, 12288)])
def test_attention_takes_slices_of_one_buffer(B, q, q_stride, out, out_stride):
    """Up to the check behind it."""
    kw = dict(q=ALIGNED + 2 * q, out=ALIGNED + 2 * out, q_stride=q_stride, out_stride=out_stride, ws_bytes=0)
    assert B.load().kvcomp_paged_attn_decode(_config(B), _memory(B), _batch(B), *_decode_args(B, **kw)) == B.ERR_CAPACITY
    assert B.load().kvcomp_paged_attn_prefill(_config(B), _memory(B), _batch(B), *_prefill_args(B, n_tokens=3, **kw)) == B.ERR_CAPACITY


@pytest.mark.parametrize("bad", [dict(d_q_out=ALIGNED + 16), dict(d_q_out=5 * ALIGNED), dict(d_q_out=6 * ALIGNED - 16),
                                 dict(q_stride=4096, q_out_stride=8192)])
def test_append_refuses_rotated_queries_over_its_inputs(B, bad):
    kw = dict(dict(Q, d_k=5 * ALIGNED, d_v=6 * ALIGNED), **bad)
    _refused(B, B.load().kvcomp_paged_append(_config(B), _memory(B), _batch(B), _new(B, **kw), None))


def test_attention_refuses_small_workspaces_and_large_batches(B):
    lib = B.load()
    small = lib.kvcomp_paged_workspace_bytes(_config(B)) - 1
    assert lib.kvcomp_paged_attn_decode(_config(B), _memory(B), _batch(B), *_decode_args(B, ws_bytes=small)) == B.ERR_CAPACITY
    assert lib.kvcomp_paged_attn_prefill(_config(B), _memory(B), _batch(B), *_prefill_args(B, ws_bytes=small)) == B.ERR_CAPACITY
    _refused(B, lib.kvcomp_paged_attn_decode(_config(B), _memory(B), _batch(B, batch=4097), *_decode_args(B)))
    _refused(B, lib.kvcomp_paged_attn_decode(_config(B, max_pages=1 << 20), _memory(B), _batch(B, batch=256), *_decode_args(B)))


def test_nothing_to_attend_is_fine(B):
    lib = B.load()
    none = _batch(B, batch=0, d_lens=0, d_table=0, d_tails=0)
    assert lib.kvcomp_paged_attn_decode(_config(B), _memory(B), none, *_decode_args(B, q=0, out=0)) == B.OK
    assert lib.kvcomp_paged_attn_prefill(_config(B), _memory(B), none, *_prefill_args(B)) == B.OK
    assert lib.kvcomp_paged_attn_prefill(_config(B), _memory(B), _batch(B), *_prefill_args(B, n_tokens=0, q=0)) == B.OK


def test_the_binding_packs_the_structures_of_the_header(B):
    """Sizes and places of the fields, against ctypes' own layout of the same declarations."""
    for packer, kind in ((B._PAGED_CONFIG, Config), (B._PAGED_CACHE, Tensors), (B._PAGED_BATCH, Batch), (B._PAGED_NEW, New)):
        assert packer.size == C.sizeof(kind)
        n = sum(3 if name == "sections" else 1 for name, _ in kind._fields_)
        got = kind.from_buffer_copy(packer.pack(*range(1, n + 1)))
        values = []
        for name, _ in kind._fields_:
            v = getattr(got, name)
            values += list(v) if name == "sections" else [v]
        assert values == list(range(1, n + 1))
