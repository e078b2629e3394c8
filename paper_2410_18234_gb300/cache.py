"""ctypes binding of the key/value cache (C ABI in include/mds_cache.h).

`Cache` owns the device memory (a torch tensor) and checks every call's
tensors, because the C entry points take bare pointers and sizes.  All device
work runs in the CUDA kernels of libmds.so, on torch's current stream or the
one given.  A step of multi-draft decoding:

    c = cache.Cache(layers, pages, kv_heads, head_dim, max_seqs, max_pages)
    c.reserve(seqs, 1 + K * L)
    for layer in range(layers):
        c.append(layer, seqs, k, v)                    # [B][1 + K * L][kv_heads][head_dim]
        o = c.attend(layer, seqs, q, branches=K)       # [B][1 + K * L][q_heads][head_dim]
    out_tokens, accept_len, _ = verifier.verify(...)   # mds.Verifier
    c.commit(seqs, accept_len, branches=K, length=L, draft_tokens=tokens, out_tokens=out_tokens)
"""
import ctypes
import math

import torch

from . import mds
from .mds import MDS_EINVAL, MDS_ESHAPE, MDS_OK, MdsError

MDS_ST_NONFINITE, MDS_ST_TIMEOUT, MDS_ST_BADTOKEN = mds.MDS_ST_NONFINITE, mds.MDS_ST_TIMEOUT, mds.MDS_ST_BADTOKEN
MDS_ST_NOPAGES, MDS_ST_BADSEQ = 128, 256
BLOCK = 16              # MDS_CACHE_BLOCK: tokens per scale
MAX_BATCH = 1024        # MDS_CACHE_MAX_BATCH
MAX_TOKENS = 1 << 20    # MDS_CACHE_MAX_TOKENS
MAX_NODES = 16384       # MDS_CACHE_MAX_NODES
MAX_GROUP = 64          # MDS_CACHE_MAX_GROUP

# every symbol include/mds_cache.h declares
EXPORTS = ("mds_cache_bytes", "mds_cache_create", "mds_cache_state", "mds_cache_reserve", "mds_cache_append",
           "mds_cache_attend", "mds_cache_commit", "mds_cache_fork", "mds_cache_truncate", "mds_cache_free",
           "mds_cache_read", "mds_cache_status", "mds_cache_destroy")


class CacheConfig(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int), ("pages", ctypes.c_int), ("page_tokens", ctypes.c_int),
                ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("max_seqs", ctypes.c_int),
                ("max_pages", ctypes.c_int), ("dtype", ctypes.c_int)]


def _bind(lib):
    vp, i, i64p = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_int64)
    cfg = ctypes.POINTER(CacheConfig)
    types = {
        "mds_cache_bytes": [cfg],
        "mds_cache_create": [ctypes.POINTER(vp), cfg, i, vp, vp],
        "mds_cache_state": [vp, ctypes.POINTER(vp), ctypes.POINTER(vp)],
        "mds_cache_reserve": [vp, vp, vp, i, i, vp],
        "mds_cache_append": [vp, i, vp, vp, vp, i64p, vp, i64p, i, i, vp],
        "mds_cache_attend": [vp, i, vp, vp, vp, i64p, vp, i, i, i, i, i, ctypes.c_float, i, vp],
        "mds_cache_commit": [vp, vp, vp, vp, vp, i, i, i, vp],
        "mds_cache_fork": [vp, vp, vp, i, vp],
        "mds_cache_truncate": [vp, vp, vp, i, vp],
        "mds_cache_free": [vp, vp, i, vp],
        "mds_cache_read": [vp, i, vp, vp, vp, vp, vp, i, i, vp],
        "mds_cache_status": [vp, ctypes.POINTER(ctypes.c_char_p)],
        "mds_cache_destroy": [vp],
    }
    for name, args in types.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.mds_cache_bytes.restype = ctypes.c_size_t
    lib.mds_cache_destroy.restype = None
    return lib


_lib = _bind(mds._lib)
_I64x3 = ctypes.c_int64 * 3


def _sizes(*given):
    """`given` as integers that the C interface's 32 bits hold: ctypes would cut larger ones."""
    out = [int(x) for x in given]
    for x in out:
        if not -1 << 31 <= x < 1 << 31:
            raise MdsError(MDS_ESHAPE, f"a size of {x}")
    return out


def _config(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens, dtype):
    return CacheConfig(*_sizes(layers, pages, page_tokens, kv_heads, head_dim, max_seqs, max_pages,
                               mds.DTYPES[dtype] if isinstance(dtype, str) else dtype))


def cache_bytes(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens=64, dtype="bf16"):
    """Device bytes of such a cache (MdsError for a configuration outside the limits)."""
    cfg = _config(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens, dtype)
    n = _lib.mds_cache_bytes(ctypes.byref(cfg))
    if n == 0:
        raise MdsError(MDS_ESHAPE, "mds_cache_bytes")
    return n


class Cache:
    """A paged key/value cache in 8 bits, with the attention that reads it.

    ``layers`` x ``pages`` pages of ``page_tokens`` (16, 32, 64 or 128) tokens
    with ``kv_heads`` heads of ``head_dim`` (64 or 128) dimensions; up to
    ``max_seqs`` sequences of ``max_pages`` pages.  ``dtype`` ("bf16" or
    "f32") is the type of keys, values, queries and outputs.

    ``seqs`` arguments are int32 CUDA tensors [B] of sequence ids, none twice
    (below 0: an unused place); ``counts`` optional int32 CUDA tensors [B].
    """

    def __init__(self, layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens=64, dtype="bf16", device=0):
        self.device = torch.device("cuda", device)
        self._index = int(device)
        self.layers, self.pages, self.page_tokens = int(layers), int(pages), int(page_tokens)
        self.kv_heads, self.head_dim = int(kv_heads), int(head_dim)
        self.max_seqs, self.max_pages = int(max_seqs), int(max_pages)
        self.ctx = None
        cfg = _config(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens, dtype)
        if cfg.dtype not in mds.TORCH_DTYPES:
            raise MdsError(MDS_EINVAL, "mds_cache_create")
        self.dtype = mds.TORCH_DTYPES[cfg.dtype]
        size = _lib.mds_cache_bytes(ctypes.byref(cfg))
        if size == 0:
            raise MdsError(MDS_ESHAPE, "mds_cache_create")
        # torch aligns to 512 bytes, the cache wants 1024
        own = torch.empty(size + 1024, dtype=torch.uint8, device=self.device)
        skip = -own.data_ptr() % 1024
        self.memory = own[skip:skip + size]
        h = ctypes.c_void_p()
        rc = _lib.mds_cache_create(ctypes.byref(h), ctypes.byref(cfg), self.device.index, self.memory.data_ptr(),
                                   self._stream(None))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_create")
        self.ctx = h
        lens, table = ctypes.c_void_p(), ctypes.c_void_p()
        _lib.mds_cache_state(h, ctypes.byref(lens), ctypes.byref(table))

        def view(ptr, *shape):
            at = ptr.value - self.memory.data_ptr()
            return self.memory[at:at + 4 * math.prod(shape)].view(torch.int32).view(shape)

        #: committed tokens [max_seqs] and page ids [max_seqs][max_pages], int32 views for reading
        self.lens = view(lens, self.max_seqs)
        self.table = view(table, self.max_seqs, self.max_pages)

    # ------------------------------------------------------------ checks

    def _stream(self, stream):
        if stream is None:
            return torch.cuda.current_stream(self.device).cuda_stream
        return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)

    def _ints(self, name, t, shape):
        """Address of an int32 tensor of this shape on the cache's device."""
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.get_device() != self._index or not t.is_contiguous():
            raise MdsError(MDS_EINVAL, f"{name}: contiguous int32 on {self.device}, got {t.dtype} on {t.device}")
        if t.shape != shape:
            raise MdsError(MDS_ESHAPE, f"{name} has shape {tuple(t.shape)}, expected {shape}")
        return t.data_ptr()

    def _seqs(self, seqs):
        if seqs.dim() != 1:
            raise MdsError(MDS_ESHAPE, f"seqs has shape {tuple(seqs.shape)}, expected (B,)")
        B = seqs.shape[0]
        return self._ints("seqs", seqs, (B,)), B

    def _rows(self, name, t, B, heads=None):
        """Check [B][n][heads][head_dim] of any strides but the last; strides of the first three axes."""
        if t.dtype is not self.dtype or t.get_device() != self._index:
            raise MdsError(MDS_EINVAL, f"{name}: {self.dtype} on {self.device}, got {t.dtype} on {t.device}")
        s = t.shape
        if len(s) != 4 or s[0] != B or s[3] != self.head_dim or (heads is not None and s[2] != heads) or \
                max(s) >= 1 << 31:
            raise MdsError(MDS_ESHAPE, f"{name} has shape {tuple(s)}, expected ({B}, n, "
                                       f"{'q_heads' if heads is None else heads}, {self.head_dim})")
        st = t.stride()
        if st[3] != 1:
            raise MdsError(MDS_EINVAL, f"{name}: the last axis must be contiguous")
        return _I64x3(*(st[i] if s[i] > 1 else 0 for i in range(3)))   # an axis of one has any stride

    def _outs(self, shape, stream, given, n=1):
        """`given`, checked, or new tensors, allocated on the stream that writes them."""
        if given is not None:
            for t in given:
                if tuple(t.shape) != shape:
                    raise MdsError(MDS_ESHAPE, f"out has shape {tuple(t.shape)}, expected {shape}")
                if t.dtype is not self.dtype or t.get_device() != self._index or not t.is_contiguous():
                    raise MdsError(MDS_EINVAL, f"out: contiguous {self.dtype} on {self.device}")
            return given
        if isinstance(stream, torch.cuda.Stream):
            with torch.cuda.stream(stream):
                return tuple(torch.empty(shape, dtype=self.dtype, device=self.device) for _ in range(n))
        got = tuple(torch.empty(shape, dtype=self.dtype, device=self.device) for _ in range(n))
        if stream is not None:
            for t in got:
                t.record_stream(torch.cuda.ExternalStream(int(stream), device=self.device))
        return got

    # ------------------------------------------------------------- calls

    def reserve(self, seqs, n, counts=None, stream=None):
        """Room for counts (n) tokens behind the committed ones of every sequence."""
        ids, B = self._seqs(seqs)
        n, = _sizes(n)
        rc = _lib.mds_cache_reserve(self.ctx, ids, self._ints("counts", counts, (B,)), n, B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_reserve")

    def append(self, layer, seqs, k, v, counts=None, stream=None):
        """Store keys and values [B][n][kv_heads][head_dim] (strided views with
        16-byte rows) in the reserved slots behind the committed tokens."""
        ids, B = self._seqs(seqs)
        ks, vs = self._rows("k", k, B, self.kv_heads), self._rows("v", v, B, self.kv_heads)
        if k.shape != v.shape:
            raise MdsError(MDS_ESHAPE, f"k has shape {tuple(k.shape)}, v {tuple(v.shape)}")
        layer, = _sizes(layer)
        rc = _lib.mds_cache_append(self.ctx, layer, ids, self._ints("counts", counts, (B,)), k.data_ptr(), ks,
                                   v.data_ptr(), vs, k.shape[1], B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_append")

    def attend(self, layer, seqs, q, branches=1, counts=None, window=0, sinks=0, scale=None, out=None, stream=None):
        """Attention of the nodes of every sequence's tree: q is
        [B][1 + branches * L][q_heads][head_dim] (a strided view with 16-byte
        rows), the result has its shape.  ``window`` and ``sinks``: 0 turns
        the window off; ``scale`` defaults to head_dim ** -0.5."""
        ids, B = self._seqs(seqs)
        qs = self._rows("q", q, B)
        layer, branches, window, sinks = _sizes(layer, branches, window, sinks)
        o, = self._outs(tuple(q.shape), stream, None if out is None else (out,))
        rc = _lib.mds_cache_attend(self.ctx, layer, ids, self._ints("counts", counts, (B,)), q.data_ptr(), qs,
                                   o.data_ptr(), q.shape[2], q.shape[1], branches, window, sinks,
                                   self.head_dim ** -0.5 if scale is None else float(scale), B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_attend")
        return o

    def commit(self, seqs, accept_len, branches=1, length=0, draft_tokens=None, out_tokens=None, stream=None):
        """Keep the root and the first accept_len tokens (-1: nothing) of the
        lowest branch whose draft_tokens [B][branches][length] are out_tokens
        [B][length + 1] (both None: branch 0); give the pages behind back."""
        ids, B = self._seqs(seqs)
        K, L = _sizes(branches, length)
        rc = _lib.mds_cache_commit(self.ctx, ids, self._ints("accept_len", accept_len, (B,)),
                                   self._ints("draft_tokens", draft_tokens, (B, K, L)),
                                   self._ints("out_tokens", out_tokens, (B, L + 1)), K, L, B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_commit")

    def fork(self, src, dst, stream=None):
        """Let the empty sequences dst share src's pages (src may name one several times)."""
        ids, B = self._seqs(src)
        rc = _lib.mds_cache_fork(self.ctx, ids, self._ints("dst", dst, (B,)), B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_fork")

    def truncate(self, seqs, lens, stream=None):
        """Shorten sequences to lens tokens and give back what is behind, reserved slots too."""
        ids, B = self._seqs(seqs)
        rc = _lib.mds_cache_truncate(self.ctx, ids, self._ints("lens", lens, (B,)), B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_truncate")

    def free(self, seqs, stream=None):
        """Empty sequences and give their pages back."""
        ids, B = self._seqs(seqs)
        rc = _lib.mds_cache_free(self.ctx, ids, B, self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_free")

    def read(self, layer, seqs, start, n, counts=None, out=None, stream=None):
        """The values of n tokens from slot start [B] (None: 0) on: k and v
        [B][n][kv_heads][head_dim], with a leading [layers] for layer None;
        zeros beyond counts and beyond what a sequence holds."""
        ids, B = self._seqs(seqs)
        n, at = _sizes(n, -1 if layer is None else layer)
        if layer is not None and at < 0:   # -1 is the C entry's name for all layers
            raise MdsError(MDS_ESHAPE, f"layer {at}")
        shape = (B, n, self.kv_heads, self.head_dim)
        if layer is None:
            shape = (self.layers, *shape)
        k, v = self._outs(shape, stream, out, 2)
        rc = _lib.mds_cache_read(self.ctx, at, ids, self._ints("start", start, (B,)),
                                 self._ints("counts", counts, (B,)), k.data_ptr(), v.data_ptr(), n, B,
                                 self._stream(stream))
        if rc != MDS_OK:
            raise MdsError(rc, "mds_cache_read")
        return k, v

    def status(self):
        """(bits, message): synchronises, reads and clears the status word."""
        msg = ctypes.c_char_p()
        rc = _lib.mds_cache_status(self.ctx, ctypes.byref(msg))
        if rc < 0:
            raise MdsError(rc, "mds_cache_status")
        return rc, (msg.value or b"").decode()

    def close(self):
        if self.ctx:
            _lib.mds_cache_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
