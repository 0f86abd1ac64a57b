"""Thin ctypes binding over libkvcomp.so (argument marshalling only; every step runs in the HIP kernels).

PyTorch is used for device memory and streams.  The library must have been built (paper_2509_00579_amd/build.py or
__graft_entry__.build()); importing this module without it raises.
"""
from __future__ import annotations

import ctypes as C
import os
import pathlib
import struct

import numpy as np
import torch

HERE = pathlib.Path(__file__).resolve().parent
LIB_PATH = HERE / "libkvcomp.so"

K, V = 0, 1
D, BT = 128, 64

OK, ERR_INVALID_ARG, ERR_STATE, ERR_CAPACITY, ERR_HIP, ERR_NONFINITE = 0, -1, -2, -3, -4, -5


class Config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32), ("head_dim", C.c_int32),
                ("block_tokens", C.c_int32), ("max_seq", C.c_int32), ("rel_eb_k", C.c_float), ("rel_eb_v", C.c_float),
                ("k_mode", C.c_int32), ("max_code_len", C.c_int32), ("buffer_tokens", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "n_blocks", "n_res", "raw_bytes", "record_bytes_k", "record_bytes_v", "header_bytes", "offsets_bytes",
        "residual_bytes", "payload_bits_k", "payload_bits_v", "stored_bytes", "max_record_bytes")] + [
        ("compression_ratio", C.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


# The paged cache's structures as packed bytes (native sizes and alignment): cheaper to make anew for every call than ctypes
# structures, and a call's arguments stay its own when several threads call.
_I32 = torch.int32
_PAGED_CONFIG = struct.Struct("@8i")          # n_kv_heads n_q_heads head_dim data_type code_type n_pages n_tails max_pages
_PAGED_CACHE = struct.Struct("@6P")           # k_codes v_codes scales k_tail v_tail fault
_PAGED_BATCH = struct.Struct("@i3P")          # batch lens table tails
_PAGED_NEW = struct.Struct("@i3P2N2P2NP4i3iP")  # n_tokens starts k v k_stride v_stride q q_out q_stride q_out_stride cos_sin
#                                               n_positions rot_dim interleaved n_axes sections positions


# every symbol include/kvcomp.h declares: name -> (restype, argtypes)
_vp, _i, _f = C.c_void_p, C.c_int, C.c_float
_cfgp = C.POINTER(Config)
SIGNATURES = {
    "kvcomp_arena_bytes": (C.c_size_t, [_cfgp]),
    "kvcomp_create": (_i, [_cfgp, _vp, C.c_size_t, _vp, C.POINTER(_vp)]),
    "kvcomp_destroy": (_i, [_vp]),
    "kvcomp_reset": (_i, [_vp, _i, _vp]),
    "kvcomp_build_codebook": (_i, [_vp, _vp, _vp, _i, _vp]),
    "kvcomp_compress_blocks": (_i, [_vp, _vp, _vp, _i, _vp]),
    "kvcomp_prefill_workspace_bytes": (C.c_size_t, [_cfgp, _i]),
    "kvcomp_prefill": (_i, [_vp, _vp, _vp, _i, _vp, C.c_size_t, _vp]),
    "kvcomp_append_token": (_i, [_vp, _vp, _vp, _vp]),
    "kvcomp_attn_decode": (_i, [_vp, _vp, _f, _vp, _vp]),
    "kvcomp_append_attn_decode": (_i, [_vp, _vp, _vp, _vp, _f, _vp, _vp]),
    "kvcomp_get_stats": (_i, [_vp, C.POINTER(Stats), _vp]),
    "kvcomp_debug_codes": (_i, [_vp, _i, _vp, _i, _vp, C.c_size_t, _vp, _vp, _vp]),
    "kvcomp_get_histogram": (_i, [_vp, _i, _vp, _vp]),
    "kvcomp_get_codebook": (_i, [_vp, _i, _vp, _vp]),
    "kvcomp_get_block_entry": (_i, [_vp, _i, _i, _i, _i, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32), _vp]),
    "kvcomp_get_block": (_i, [_vp, _i, _i, _i, _i, _vp, C.c_size_t, C.POINTER(C.c_size_t), _vp]),
    "kvcomp_get_residual": (_i, [_vp, _i, _vp, C.POINTER(_i), _vp]),
    "kvcomp_decompress": (_i, [_vp, _i, _vp, _i, _vp]),
    "kvcomp_decompress_tree_walk": (_i, [_vp, _i, _vp, _i, _vp]),
    "kvcomp_set_tuning": (_i, [_vp, _i, _i, _i]),
    "kvcomp_set_profiling": (_i, [_vp, _i]),
    "kvcomp_get_profile": (_i, [_vp, C.POINTER(_i), C.POINTER(C.c_double)]),
    "kvcomp_probe_read_stream": (_i, [_vp, C.c_size_t, _vp, C.POINTER(C.c_size_t), _vp]),
    "kvcomp_baseline_workspace_bytes": (C.c_size_t, [_cfgp]),
    "kvcomp_baseline_fp16_attn": (_i, [_cfgp, _vp, _vp, _i, _vp, _f, _vp, _vp, C.c_size_t, _i, _vp]),
    "kvcomp_baseline_fp16_attn_noalloc": (_i, [_cfgp, _vp, _vp, _i, _vp, _f, _vp, _i, _vp]),
    "kvcomp_paged_append": (_i, [_vp, _vp, _vp, _vp, _vp]),
    "kvcomp_paged_workspace_bytes": (C.c_size_t, [_vp]),
    "kvcomp_paged_attn_decode": (_i, [_vp, _vp, _vp, _vp, C.c_size_t, _i, _f, _i, _i, _vp, C.c_size_t, _vp, C.c_size_t, _vp]),
    "kvcomp_paged_attn_prefill": (_i, [_vp, _vp, _vp, _vp, C.c_size_t, _vp, _i, _f, _i, _i, _i, _vp, C.c_size_t, _vp,
                                       C.c_size_t, _vp]),
    "kvcomp_paged_check": (_i, [_vp, _vp]),
    "kvcomp_last_error": (C.c_char_p, []),
}

_lib = None


def load():
    """Load libkvcomp.so; fails loudly when the HIP extension has not been built."""
    global _lib
    if _lib is None:
        path = pathlib.Path(os.environ.get("KVCOMP_LIB", LIB_PATH))  # KVCOMP_LIB: try another build of the library
        if not path.exists():
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2509_00579_amd.build` "
                               "(there is no CPU fallback)")
        lib = C.CDLL(str(path))
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


class KvcompError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"kvcomp status {status}: {msg}")
        self.status = status


def _check(st):
    if st != OK:
        raise KvcompError(st, load().kvcomp_last_error().decode())


# A decode step of a short cache takes 8 us on the GPU, so what a call costs on the host shows: the raw stream handle instead
# of a torch.cuda.Stream object (0.3 instead of 4 us), plain integers for ctypes' pointer arguments, no tuples made anew.
def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev_fp16(t, shape):
    assert t.is_cuda and t.dtype is torch.float16 and t.is_contiguous(), "expected a contiguous CUDA fp16 tensor"
    assert t.shape == shape, f"expected shape {tuple(shape)}, got {tuple(t.shape)}"
    return t.data_ptr()


def _dev_out(t):
    assert t.is_cuda and t.dtype is torch.float32 and t.is_contiguous()
    return t.data_ptr()


def make_config(batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, k_mode=0, max_code_len=0,
                buffer_tokens=0):
    return Config(batch, n_kv_heads, n_q_heads, D, BT, max_seq, rel_eb_k, rel_eb_v, k_mode, max_code_len,
                  buffer_tokens)


class KVCompCache:
    """One layer's compressed KV cache on the GPU: the four calls of the hot path plus the parity exports."""

    def __init__(self, batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, k_mode=0, max_code_len=0,
                 buffer_tokens=0, device="cuda:0", arena=None):
        self.lib = load()
        self.cfg = make_config(batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, k_mode, max_code_len,
                               buffer_tokens)
        self.buffer_tokens = buffer_tokens or BT
        self.B, self.H, self.Hq, self.max_seq = batch, n_kv_heads, n_q_heads, max_seq
        self.device = torch.device(device)
        nbytes = self.lib.kvcomp_arena_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise KvcompError(ERR_INVALID_ARG, "invalid configuration")
        if arena is None:
            arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        assert arena.is_cuda and arena.dtype == torch.uint8 and arena.is_contiguous() and arena.numel() >= nbytes
        assert arena.data_ptr() % 256 == 0
        self.arena = arena
        h = C.c_void_p()
        _check(self.lib.kvcomp_create(C.byref(self.cfg), C.c_void_p(self.arena.data_ptr()), nbytes, _stream(), C.byref(h)))
        self.h = h
        self._token_shape, self._q_shape = (batch, n_kv_heads, D), (batch, n_q_heads, D)

    def close(self):
        if getattr(self, "h", None):
            self.lib.kvcomp_destroy(self.h)
            self.h = None

    __del__ = close

    # ---- hot path ----
    def build_codebook(self, Kt, Vt):
        S = Kt.shape[1]
        shape = (self.B, S, self.H, D)
        _check(self.lib.kvcomp_build_codebook(self.h, _dev_fp16(Kt, shape), _dev_fp16(Vt, shape), S, _stream()))

    def compress_blocks(self, Kt, Vt):
        S = Kt.shape[1]
        shape = (self.B, S, self.H, D)
        _check(self.lib.kvcomp_compress_blocks(self.h, _dev_fp16(Kt, shape), _dev_fp16(Vt, shape), S, _stream()))

    def prefill_workspace_bytes(self, S):
        return self.lib.kvcomp_prefill_workspace_bytes(C.byref(self.cfg), S)

    def prefill(self, Kt, Vt, workspace=None):
        """build_codebook + compress_blocks with one quantization pass; `workspace`: a uint8 CUDA tensor of at least
        prefill_workspace_bytes(S) bytes (allocated here if None)."""
        S = Kt.shape[1]
        shape = (self.B, S, self.H, D)
        if workspace is None:
            workspace = torch.empty(self.prefill_workspace_bytes(S), dtype=torch.uint8, device=self.device)
        assert workspace.is_cuda and workspace.dtype == torch.uint8 and workspace.is_contiguous()
        _check(self.lib.kvcomp_prefill(self.h, _dev_fp16(Kt, shape), _dev_fp16(Vt, shape), S,
                                       C.c_void_p(workspace.data_ptr()), workspace.numel(), _stream()))

    def append_token(self, k_new, v_new):
        shape = self._token_shape
        _check(self.lib.kvcomp_append_token(self.h, _dev_fp16(k_new, shape), _dev_fp16(v_new, shape), _stream()))

    def attn_decode(self, q, scale, out=None):
        if out is None:
            out = torch.empty(self._q_shape, dtype=torch.float32, device=self.device)
        _check(self.lib.kvcomp_attn_decode(self.h, _dev_fp16(q, self._q_shape), float(scale), _dev_out(out), _stream()))
        return out

    def append_attn_decode(self, k_new, v_new, q, scale, out=None):
        """append_token followed by attn_decode, in one launch whenever no block has to be compressed."""
        if out is None:
            out = torch.empty(self._q_shape, dtype=torch.float32, device=self.device)
        shape = self._token_shape
        _check(self.lib.kvcomp_append_attn_decode(self.h, _dev_fp16(k_new, shape), _dev_fp16(v_new, shape),
                                                  _dev_fp16(q, self._q_shape), float(scale), _dev_out(out), _stream()))
        return out

    def reset(self, keep_codebook=True):
        _check(self.lib.kvcomp_reset(self.h, int(keep_codebook), _stream()))

    # ---- metrics / parity exports ----
    def stats(self):
        st = Stats()
        _check(self.lib.kvcomp_get_stats(self.h, C.byref(st), _stream()))
        return st.as_dict()

    def debug_codes(self, which, X):
        S = X.shape[1]
        nblk = self.B * self.H * (S // BT)
        units = (1 if self.cfg.k_mode == 1 else D) if which == K else BT
        scratch = torch.empty(nblk * (BT * D + 4 * units), dtype=torch.uint8, device=self.device)
        codes = np.zeros((nblk, BT, D), np.uint8)
        mm = np.zeros((nblk, units, 2), np.uint16)
        _check(self.lib.kvcomp_debug_codes(self.h, which, _dev_fp16(X, (self.B, S, self.H, D)), S,
                                           C.c_void_p(scratch.data_ptr()), scratch.numel(),
                                           codes.ctypes.data_as(C.c_void_p), mm.ctypes.data_as(C.c_void_p), _stream()))
        return codes, mm

    def histogram(self, which):
        h = np.zeros(256, np.uint32)
        _check(self.lib.kvcomp_get_histogram(self.h, which, h.ctypes.data_as(C.c_void_p), _stream()))
        return h

    def codebook(self, which):
        ln, cd = np.zeros(256, np.uint8), np.zeros(256, np.uint32)
        _check(self.lib.kvcomp_get_codebook(self.h, which, ln.ctypes.data_as(C.c_void_p), cd.ctypes.data_as(C.c_void_p)))
        return ln, cd

    def block_entry(self, which, b, h, blk):
        o, s = C.c_uint32(), C.c_uint32()
        _check(self.lib.kvcomp_get_block_entry(self.h, which, b, h, blk, C.byref(o), C.byref(s), _stream()))
        return o.value, s.value

    def get_block(self, which, b, h, blk):
        buf = np.zeros(16384, np.uint8)
        n = C.c_size_t()
        _check(self.lib.kvcomp_get_block(self.h, which, b, h, blk, buf.ctypes.data_as(C.c_void_p), buf.size, C.byref(n),
                                         _stream()))
        return buf[: n.value].copy()

    def residual(self, which):
        buf = np.zeros((self.B, self.buffer_tokens, self.H, D), np.uint16)
        n = C.c_int()
        _check(self.lib.kvcomp_get_residual(self.h, which, buf.ctypes.data_as(C.c_void_p), C.byref(n), _stream()))
        return buf.view(np.float16)[:, : n.value], n.value

    def decompress(self, which, tokens, out=None, tree_walk=False):
        """The cache of one tensor as fp16 [B, tokens, H, 128] (stand-alone decompression; tree_walk: with the
        bit-serial decoder instead of the table decoder)."""
        if out is None:
            out = torch.empty((self.B, tokens, self.H, D), dtype=torch.float16, device=self.device)
        assert out.is_cuda and out.is_contiguous() and out.dtype == torch.float16
        fn = self.lib.kvcomp_decompress_tree_walk if tree_walk else self.lib.kvcomp_decompress
        _check(fn(self.h, which, C.c_void_p(out.data_ptr()), int(out.shape[1]), _stream()))
        return out

    def set_tuning(self, n_splits=0, stage_bytes=0, waves=0):
        _check(self.lib.kvcomp_set_tuning(self.h, n_splits, stage_bytes, waves))

    def set_profiling(self, enable):
        _check(self.lib.kvcomp_set_profiling(self.h, int(enable)))

    def get_profile(self):
        n, ms = C.c_int(), C.c_double()
        _check(self.lib.kvcomp_get_profile(self.h, C.byref(n), C.byref(ms)))
        return n.value, ms.value


class KVCompLayers:
    """The caches of all layers of a model: one context per layer (Section 3: buffers and codebooks are per layer,
    the K and the V codebook of a layer are built from that layer's prompt), carved out of a single device
    allocation.  `layers[i]` is the KVCompCache of layer i; nothing is computed here."""

    def __init__(self, n_layers, batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, device="cuda:0", **kw):
        lib = load()
        cfg = make_config(batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, kw.get("k_mode", 0),
                          kw.get("max_code_len", 0), kw.get("buffer_tokens", 0))
        per_layer = lib.kvcomp_arena_bytes(C.byref(cfg))
        if per_layer == 0 or n_layers < 1:
            raise KvcompError(ERR_INVALID_ARG, "invalid configuration")
        per_layer = (per_layer + 255) // 256 * 256
        self.arena = torch.empty(n_layers * per_layer, dtype=torch.uint8, device=torch.device(device))
        self.layers = [KVCompCache(batch, n_kv_heads, n_q_heads, max_seq, rel_eb_k, rel_eb_v, device=device,
                                   arena=self.arena[i * per_layer:(i + 1) * per_layer], **kw) for i in range(n_layers)]

    def __len__(self):
        return len(self.layers)

    def __getitem__(self, i):
        return self.layers[i]

    def stats(self):
        """Byte counts summed over the layers, and the overall compression ratio."""
        per = [c.stats() for c in self.layers]
        tot = {k: sum(p[k] for p in per) for k in ("raw_bytes", "record_bytes_k", "record_bytes_v", "header_bytes",
                                                    "offsets_bytes", "residual_bytes", "stored_bytes")}
        tot["compression_ratio"] = tot["raw_bytes"] / tot["stored_bytes"] if tot["stored_bytes"] else 0.0
        return tot

    def close(self):
        for c in self.layers:
            c.close()


def probe_read_stream(buf, sink):
    """One plain streaming read of the uint8 CUDA tensor `buf` (measurement aid); returns the bytes it reads."""
    assert buf.is_cuda and buf.is_contiguous() and sink.is_cuda and sink.numel() * sink.element_size() >= 4
    n = C.c_size_t()
    _check(load().kvcomp_probe_read_stream(C.c_void_p(buf.data_ptr()), buf.numel() * buf.element_size(),
                                           C.c_void_p(sink.data_ptr()), C.byref(n), _stream()))
    return n.value


class BaselineFp16Attention:
    """Decode attention on the uncompressed fp16 cache (the comparison kernel)."""

    def __init__(self, batch, n_kv_heads, n_q_heads, device="cuda:0"):
        self.lib = load()
        self.cfg = make_config(batch, n_kv_heads, n_q_heads, 64, 0.01, 0.01)
        self.B, self.H, self.Hq = batch, n_kv_heads, n_q_heads
        self.device = torch.device(device)
        self.ws = torch.zeros(self.lib.kvcomp_baseline_workspace_bytes(C.byref(self.cfg)), dtype=torch.uint8,
                              device=self.device)  # zero-filled once: it holds the split tickets

    def __call__(self, Kt, Vt, q, scale, out=None, n_splits=0):
        S = Kt.shape[1]
        shape = (self.B, S, self.H, D)
        if out is None:
            out = torch.empty((self.B, self.Hq, D), dtype=torch.float32, device=self.device)
        _check(self.lib.kvcomp_baseline_fp16_attn(C.byref(self.cfg), _dev_fp16(Kt, shape), _dev_fp16(Vt, shape), S,
                                                  _dev_fp16(q, (self.B, self.Hq, D)), float(scale),
                                                  C.c_void_p(out.data_ptr()), C.c_void_p(self.ws.data_ptr()),
                                                  self.ws.numel(), n_splits, _stream()))
        return out

    def noalloc(self, Kt, Vt, q, scale, out, n_splits=0):
        """The same through kvcomp_baseline_fp16_attn_noalloc: no workspace, the library's static scratch; `out` is
        the caller's."""
        S = Kt.shape[1]
        shape = (self.B, S, self.H, D)
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous()
        _check(self.lib.kvcomp_baseline_fp16_attn_noalloc(C.byref(self.cfg), _dev_fp16(Kt, shape), _dev_fp16(Vt, shape), S,
                                                          _dev_fp16(q, (self.B, self.Hq, D)), float(scale),
                                                          C.c_void_p(out.data_ptr()), n_splits, _stream()))
        return out


# looked up once: the calls of a step are short
_current_device, _raw_stream = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


class Rope:
    """The position rotation of PagedCache.append: `cos_sin` is a CUDA fp32 tensor [positions, rot_dim], the cosines of the
    rot_dim / 2 pairs and then their sines; interleaved: pairs are neighbouring channels instead of the two halves of the
    rotated ones; sections: pairs per position axis (time, height, width), one axis if None."""

    def __init__(self, cos_sin, interleaved=False, sections=None):
        assert cos_sin.is_cuda and cos_sin.dtype is torch.float32 and cos_sin.is_contiguous() and cos_sin.dim() == 2
        self.cos_sin = cos_sin
        self.n_positions, self.rot_dim = cos_sin.shape
        sections = [self.rot_dim // 2] if sections is None else list(sections)
        assert 1 <= len(sections) <= 3, "one to three axes"
        self.interleaved, self.n_axes = int(interleaved), len(sections)
        self.sections = tuple(sections) + (0,) * (3 - len(sections))

    @staticmethod
    def table(n_positions, rot_dim, base=10000.0, device="cuda:0"):
        """The usual table: the angle of pair p at position n is n * base^(-2p / rot_dim), taken in 64 bits."""
        half = rot_dim // 2
        angle = torch.arange(n_positions, device=device, dtype=torch.float64)[:, None] * base ** (
            -torch.arange(half, device=device, dtype=torch.float64) / half)
        return torch.cat([angle.cos(), angle.sin()], dim=1).float()


class PagedCache:
    """One layer's paged KV cache of 8-bit codes for sequences of different lengths (the layout stands in include/kvcomp.h).

    The pages, scales and tails are tensors of the caller's, `storage` = (k_codes, v_codes, scales, k_tail, v_tail), or are
    allocated here.  Which sequence has which pages and tail, and how long it is, comes with every call: lens [batch], table
    [batch, max_pages] and tails [batch] are int32 CUDA tensors, read on the device.  lens counts the call's own tokens.
    `workspace` is the attention calls' scratch (69 MB for heads of 128, 36 MB for 64), a cache's own if None; caches whose calls
    never overlap in time (the layers of a model on one stream) may share one, and do well to; calls on several streams at a time
    need one each (new_workspace).  What the cache allocated itself, new_workspace's tensors too, may be used on any stream, and
    let go while calls are still running; the caller's tensors are the caller's to keep."""

    def __init__(self, n_kv_heads, n_q_heads, n_pages, n_tails, head_dim=D, dtype=torch.float16, codes="int8", device="cuda:0",
                 storage=None, workspace=None):
        self.lib = load()
        self._append, self._decode, self._prefill = (self.lib.kvcomp_paged_append, self.lib.kvcomp_paged_attn_decode,
                                                     self.lib.kvcomp_paged_attn_prefill)
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.H, self.Hq, self.D, self.dtype = n_kv_heads, n_q_heads, head_dim, dtype
        self.n_pages, self.n_tails = n_pages, n_tails
        code = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}[codes]
        kinds = (("k_codes", (n_pages, n_kv_heads, BT, head_dim), code), ("v_codes", (n_pages, n_kv_heads, head_dim, BT), code),
                 ("scales", (n_pages, n_kv_heads, 2), torch.float32), ("k_tail", (n_tails, n_kv_heads, BT, head_dim), dtype),
                 ("v_tail", (n_tails, n_kv_heads, BT, head_dim), dtype))
        self._own = []
        if storage is None:
            storage = self._own = [torch.empty(shape, dtype=t, device=self.device) for _, shape, t in kinds]
        for (name, shape, t), x in zip(kinds, storage):
            assert x.device == self.device and x.dtype is t and x.is_contiguous() and x.shape == shape, (
                f"{name} must be a contiguous {t} tensor {shape} on {self.device}")
            setattr(self, name, x)
        self.fault = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._types = (head_dim, {torch.float16: 0, torch.bfloat16: 1}[dtype], int(codes == "e4m3"), n_pages, n_tails)
        self._memory = _PAGED_CACHE.pack(*(x.data_ptr() for x in (*storage, self.fault)))
        self._index = self.device.index
        self._config = {}
        self._streams = {_raw_stream(self._index)}  # that the allocator knows the cache's own tensors on
        self._own = [*self._own, self.fault]
        self._workspace = self._scratch(self.new_workspace() if workspace is None else workspace, _raw_stream(self._index))
        self._settle()

    def _cfg(self, max_pages):
        cfg = self._config.get(max_pages)
        if cfg is None:
            cfg = self._config[max_pages] = _PAGED_CONFIG.pack(self.H, self.Hq, *self._types, max_pages)
        return cfg

    def _batch(self, lens, table, tails):
        """The packed sequences, their number and the configuration that goes with the table's width."""
        shape, wide = lens.shape, table.shape
        assert lens.dtype is _I32 and table.dtype is _I32 and tails.dtype is _I32, "lens, table and tails are int32"
        assert lens.get_device() == table.get_device() == tails.get_device() == self._index, f"lens, table and tails must be on {self.device}"
        assert len(shape) == 1 and tails.shape == shape and len(wide) == 2 and wide[0] == shape[0], "one row per sequence"
        assert table.is_contiguous() and lens.is_contiguous() and tails.is_contiguous(), "lens, table and tails must be contiguous"
        return _PAGED_BATCH.pack(shape[0], lens.data_ptr(), table.data_ptr(), tails.data_ptr()), shape[0], self._cfg(wide[1])

    def _starts(self, starts, batch):
        assert starts.dtype is _I32 and starts.get_device() == self._index and starts.is_contiguous()
        assert starts.shape == (batch + 1,), "starts: one entry per sequence and the end"
        return starts.data_ptr()

    def _rows(self, x, shape, name):
        """Pointer and token stride of a tensor [n, heads, head_dim] whose tokens may be apart (a slice of a fused projection)."""
        assert x.get_device() == self._index and x.dtype is self.dtype, f"{name} must be {self.dtype} on {self.device}"
        assert x.shape == shape, f"{name}: expected shape {shape}, got {tuple(x.shape)}"
        if x.is_contiguous():
            return x.data_ptr(), shape[1] * shape[2]
        s0, s1, s2 = x.stride()
        assert s2 == 1 and (s1 == shape[2] or shape[1] == 1), f"the heads of a token of {name} must be contiguous"
        return x.data_ptr(), s0 if shape[0] > 1 else shape[1] * shape[2]

    def _on_device(self):
        if _current_device() != self._index:
            raise KvcompError(ERR_INVALID_ARG, f"the current device is not the cache's ({self.device})")
        stream = _raw_stream(self._index)
        if stream not in self._streams:
            for x in self._own:
                x.record_stream(torch.cuda.current_stream(self.device))
            self._streams.add(stream)
        return stream

    def _settle(self):
        """What was cleared on this stream is used on others."""
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.device).synchronize()

    def append(self, k, v, lens, table, tails, starts=None, q=None, q_out=None, rope=None, positions=None):
        """Append k, v [n, n_kv_heads, head_dim]: one token per sequence (starts None: n = batch), or rows starts[b] ..
        starts[b + 1] to sequence b (starts: int32 [batch + 1]).  With `rope`, keys are rotated, and queries q into q_out (which
        may be q, and is q's rotated copy if None) with them; positions: int32 [axes, n] (default: a token's place).
        Returns q_out."""
        stream = self._on_device()
        n = k.shape[0]
        seqs, batch, cfg = self._batch(lens, table, tails)
        shape = (n, self.H, self.D)
        kp, ks = self._rows(k, shape, "k")
        vp, vs = self._rows(v, shape, "v")
        sp = qp = qs = op = os_ = cp = n_pos = rot = inter = pp = 0
        axes, sections = 1, (0, 0, 0)
        if starts is not None:
            sp = self._starts(starts, batch)
        assert q is not None or q_out is None, "q_out without q"
        assert rope is not None or positions is None, "positions without rope"
        if q is not None:
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            shape = (n, self.Hq, self.D)
            qp, qs = self._rows(q, shape, "q")
            op, os_ = self._rows(q_out, shape, "q_out")
        if rope is not None:
            assert rope.cos_sin.get_device() == self._index
            cp, n_pos, rot, inter, axes, sections = (rope.cos_sin.data_ptr(), rope.n_positions, rope.rot_dim, rope.interleaved,
                                                     rope.n_axes, rope.sections)
            if positions is not None:
                assert positions.dtype is torch.int32 and positions.get_device() == self._index and positions.is_contiguous()
                assert positions.shape == (axes, n), f"positions: expected shape {(axes, n)}, got {tuple(positions.shape)}"
                pp = positions.data_ptr()
        new = _PAGED_NEW.pack(n, sp, kp, vp, ks, vs, qp, op, qs, os_, cp, n_pos, rot, inter, axes, *sections, pp)
        st = self._append(cfg, self._memory, seqs, new, stream)
        if st:
            _check(st)
        return q_out

    def new_workspace(self):
        """Scratch of the attention calls, for one of them at a time."""
        workspace = torch.zeros(self.lib.kvcomp_paged_workspace_bytes(self._cfg(1)), dtype=torch.uint8, device=self.device)
        workspace.known_streams = {_raw_stream(self._index)}  # that the allocator knows it on
        self._settle()
        return workspace

    def _scratch(self, workspace, stream):
        if workspace is None:
            workspace = self._workspace
        else:
            assert workspace.get_device() == self._index and workspace.dtype is torch.uint8 and workspace.is_contiguous()
        known = getattr(workspace, "known_streams", None)  # None: the caller's own tensor
        if known is not None and stream not in known:
            workspace.record_stream(torch.cuda.current_stream(self.device))
            known.add(stream)
        return workspace

    def attn_decode(self, q, scale, lens, table, tails, q_len=1, window=0, max_len=0, out=None, workspace=None):
        """Attention of q [batch * q_len, n_q_heads, head_dim], the last q_len tokens of every sequence, over the cache;
        window: keys that a token sees, itself included (0: all before it); max_len: the longest length, if known."""
        stream = self._on_device()
        seqs, batch, cfg = self._batch(lens, table, tails)
        shape = (batch * q_len, self.Hq, self.D)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        qp, qs = self._rows(q, shape, "q")
        op, os_ = self._rows(out, shape, "out")
        ws = self._scratch(workspace, stream)
        _check(self._decode(cfg, self._memory, seqs, qp, qs, q_len, float(scale), window, max_len, op, os_, ws.data_ptr(), ws.numel(),
                            stream))
        return out

    def attn_prefill(self, q, scale, starts, lens, table, tails, max_new=0, max_len=0, window=0, out=None, workspace=None):
        """Attention of chunks: rows starts[b] .. starts[b + 1] of q [n, n_q_heads, head_dim] are the last tokens of sequence b
        (starts: int32 [batch + 1]); max_new, max_len: the longest chunk and length, if known."""
        stream = self._on_device()
        seqs, batch, cfg = self._batch(lens, table, tails)
        sp = self._starts(starts, batch)
        n = q.shape[0]
        shape = (n, self.Hq, self.D)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        qp, qs = self._rows(q, shape, "q")
        op, os_ = self._rows(out, shape, "out")
        ws = self._scratch(workspace, stream)
        _check(self._prefill(cfg, self._memory, seqs, qp, qs, sp, n, float(scale), window, max_new, max_len, op, os_, ws.data_ptr(),
                             ws.numel(), stream))
        return out

    def check(self):
        """Raises what kernels flagged since the last check (pages out of range, Inf or NaN appended); synchronises."""
        _check(self.lib.kvcomp_paged_check(self._memory, self._on_device()))
