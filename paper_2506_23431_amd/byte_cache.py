"""A cache of keys and values in 8 bits on one GPU: the operators of include/pd.h on torch tensors (argument checks and
marshalling only; every step runs inside libpd.so)."""

import ctypes as C
import math

import torch

from .binding import PdByteCache, PdError, _check, load

BLOCK = 64                                              # PD_BYTE_BLOCK
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # PD_TYPE_*
_I64x3 = C.c_int64 * 3
# The number of the current device and the handle of its current stream, without the objects around them (3 us of a call).
_current_device = torch.cuda.current_device
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _require(ok, message, *args):
    if not ok:
        raise PdError(message % args)


class ByteCache:
    """Keys and values of n_req requests with room for max_tokens tokens each; how they are held stands at pd_byte_cache.

    How many tokens a request holds is the caller's to know and is passed to every call as `lens`, an int32 tensor [n_req] on the
    cache's device that is read when the kernels run.  Work is queued on the current stream of that device; nothing is kept
    between calls but the tensors k, v, k_scale, v_scale, k_tail, v_tail, and calls can be captured into a graph."""

    def __init__(self, n_req, n_kv_head, head_dim, max_tokens, device="cuda:0"):
        n_block = -(-max_tokens // BLOCK)
        zeros = lambda *shape, dtype: torch.zeros(*shape, dtype=dtype, device=device)  # noqa: E731
        self._hold(zeros(n_req, n_kv_head, n_block, BLOCK, head_dim, dtype=torch.int8),
                   zeros(n_req, n_kv_head, n_block, head_dim, BLOCK, dtype=torch.int8),
                   zeros(n_req, n_kv_head, n_block, dtype=torch.float32),
                   zeros(n_req, n_kv_head, n_block, dtype=torch.float32),
                   zeros(n_req, n_kv_head, 2, BLOCK, head_dim, dtype=torch.float16),
                   zeros(n_req, n_kv_head, 2, head_dim, BLOCK, dtype=torch.float16))

    @classmethod
    def from_tensors(cls, k, v, k_scale, v_scale, k_tail, v_tail):
        """A cache in tensors that are there already (not copied)."""
        self = cls.__new__(cls)
        self._hold(k, v, k_scale, v_scale, k_tail, v_tail)
        return self

    def _hold(self, k, v, k_scale, v_scale, k_tail, v_tail):
        _require(k.dim() == 5 and k.shape[3] == BLOCK, "k must be [req][head][block][%d][dim], not %s", BLOCK, tuple(k.shape))
        req, heads, n_block, _, dim = k.shape
        for name, t, shape, dtype in (("k", k, k.shape, torch.int8), ("v", v, (req, heads, n_block, dim, BLOCK), torch.int8),
                                      ("k_scale", k_scale, (req, heads, n_block), torch.float32),
                                      ("v_scale", v_scale, (req, heads, n_block), torch.float32),
                                      ("k_tail", k_tail, (req, heads, 2, BLOCK, dim), torch.float16),
                                      ("v_tail", v_tail, (req, heads, 2, dim, BLOCK), torch.float16)):
            _require(tuple(t.shape) == tuple(shape) and t.dtype == dtype, "%s must be %s %s, not %s %s", name, dtype,
                     tuple(shape), t.dtype, tuple(t.shape))
            _require(t.is_contiguous() and t.device == k.device, "%s must be contiguous and on %s", name, k.device)
        _require(dim in (32, 64, 96, 128) and min(req, heads, n_block) >= 1,
                 "a byte cache has requests, heads, blocks and heads of 32, 64, 96 or 128, not %s", tuple(k.shape))
        _require(k.device.type == "cuda", "a byte cache lives on a GPU, not on %s", k.device)
        self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail = k, v, k_scale, v_scale, k_tail, v_tail
        self.n_req, self.n_kv_head, self.n_block, self.head_dim = req, heads, n_block, dim
        self.device = k.device
        self._scale = 1.0 / math.sqrt(dim)
        self._lib = load()
        self._c = PdByteCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k_tail.data_ptr(),
                              v_tail.data_ptr(), req, heads, dim, n_block)
        self._p = C.byref(self._c)

    # -- what every call checks --------------------------------------------------
    def _data(self, name, t, shape):
        """Pointer and strides of a tensor [req][token or row][head][dim] whose dims lie together."""
        if t.shape != shape or t.device != self.device or t.dtype not in _TYPES:
            raise PdError(f"{name} must be float32, bfloat16 or float16 {shape} on {self.device}, not {t.dtype} "
                          f"{tuple(t.shape)} on {t.device}")
        st = t.stride()
        if st[3] != 1:
            raise PdError(f"the dims of {name} must lie together")
        return t.data_ptr(), _I64x3(st[0], st[1], st[2])

    def _ints(self, name, t, shape, dtype=torch.int32):
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype or t.device != self.device or not t.is_contiguous():
            raise PdError(f"{name} must be contiguous {dtype} {shape} on {self.device}, not {t.dtype} {tuple(t.shape)} on "
                          f"{t.device}")
        return t.data_ptr()

    def _call(self, function, *args):
        index = self.device.index
        if index == _current_device():
            _check(function(self._p, *args, _raw_stream(index)))
        else:
            with torch.cuda.device(index):
                _check(function(self._p, *args, _raw_stream(index)))

    # -- the operators -----------------------------------------------------------
    def append(self, k, v, lens, counts=None):
        """Stores new tokens k, v [req][new][head][dim] (fp32, bf16 or fp16) behind those that the requests hold.

        lens: int32 [req], tokens of each request with the new ones; counts: int32 [req] or None, how many are new (None: all of
        k and v; fewer: the rest is padding).  A request whose numbers do not fit is left as it is."""
        _require(k.dim() == 4, "k must be [req][new][head][dim], not %s", k.shape)
        n_new = k.shape[1]
        shape = (self.n_req, n_new, self.n_kv_head, self.head_dim)
        kp, ks = self._data("k", k, shape)
        vp, vs = self._data("v", v, shape)
        dtype = k.dtype
        _require(dtype == v.dtype, "k and v must have the same type, not %s and %s", dtype, v.dtype)
        self._call(self._lib.pd_byte_append, kp, vp, _TYPES[dtype], ks, vs, n_new,
                   self._ints("counts", counts, (self.n_req,)), self._ints("lens", lens, (self.n_req,)))

    def read(self, lens, n_tok, first=None, dtype=torch.float32):
        """Keys and values [req][n_tok][head][dim] of tokens first[r] .. first[r] + n_tok - 1 (int32 [req]; None: from 0) as the
        values that they stand for; zeros where a request holds none."""
        _require(n_tok >= 0, "n_tok must be >= 0, not %s", n_tok)
        _require(dtype in _TYPES, "dtype must be float32, bfloat16 or float16, not %s", dtype)
        both = torch.empty((2, self.n_req, n_tok, self.n_kv_head, self.head_dim), dtype=dtype, device=self.device)
        k, v = both.unbind()
        self._call(self._lib.pd_byte_read, self._ints("first", first, (self.n_req,)), n_tok,
                   self._ints("lens", lens, (self.n_req,)), k.data_ptr(), v.data_ptr(), _TYPES[dtype])
        return k, v

    def attention(self, q, lens, row_limit=None, key_tag=None, row_tag=None, scale=None, max_len=0, with_lse=False):
        """softmax(scale q k) v of query rows q [req][row][head][dim]; returns the same shape and type (and, with_lse, the
        logarithms of the sums, fp32 [req][row][head]).

        A row sees the tokens below lens[request] and, where given, below row_limit (int32 [req][row]) and with key_tag (uint16
        [req][n_block * 64]) at most row_tag (int32 [req][row]); one that sees nothing gives zeros.  head: a multiple of the
        key heads, each of which serves the query heads in turn.  scale: 1 / sqrt(dim) unless given.  max_len: a number that
        no entry of lens exceeds, if known (shorter launches)."""
        _require(q.dim() == 4, "q must be [req][row][head][dim], not %s", q.shape)
        n_req, device = self.n_req, self.device
        _, rows, heads, _ = q.shape
        qp, qs = self._data("q", q, (n_req, rows, heads, self.head_dim))
        need = self._lib.pd_byte_attention_workspace_bytes(self._p, heads, rows, max_len)
        if need == 0:
            raise PdError(f"invalid attention: {self._lib.pd_last_error().decode()}")
        out = torch.empty((n_req, rows, heads, self.head_dim), dtype=q.dtype, device=device)
        lse = torch.empty((n_req, rows, heads), dtype=torch.float32, device=device) if with_lse else None
        # of the caller's stream, or of the graph that captures it: never shared by two calls that may overlap
        work = torch.empty(need, dtype=torch.uint8, device=device) if need > 16 else None
        self._call(self._lib.pd_byte_attention, qp, _TYPES[q.dtype], qs, heads, rows, self._ints("lens", lens, (n_req,)),
                   self._ints("row_limit", row_limit, (n_req, rows)),
                   self._ints("key_tag", key_tag, (n_req, self.n_block * BLOCK), torch.uint16),
                   self._ints("row_tag", row_tag, (n_req, rows)),
                   self._scale if scale is None else scale, max_len, out.data_ptr(),
                   lse.data_ptr() if with_lse else None, work.data_ptr() if work is not None else None, need)
        return (out, lse) if with_lse else out
