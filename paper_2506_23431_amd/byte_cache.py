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
    cache's device that is read when the kernels run: the numbers that the last append was given, not a bound on what is read (for
    that there are row_limit, first and n_tok; a smaller number that ends inside a whole block finds other tokens there, or none).  Work is queued on the current stream of that device; nothing is kept
    between calls but the tensors k, v, k_scale, v_scale, k_tail, v_tail, and calls can be captured into a graph.  For inference:
    no gradients are recorded."""

    def __init__(self, n_req, n_kv_head, head_dim, max_tokens, device="cuda:0"):
        device, n_block = torch.device(device), -(-max_tokens // BLOCK)
        _require(device.type == "cuda", "a byte cache lives on a GPU, not on %s", device)
        _require(head_dim in (32, 64, 96, 128) and min(n_req, n_kv_head, n_block) >= 1,
                 "a byte cache has requests, heads and blocks, and heads of 32, 64, 96 or 128: not %s",
                 (n_req, n_kv_head, n_block, head_dim))
        zeros = lambda *shape, dtype: torch.zeros(n_req, n_kv_head, *shape, dtype=dtype, device=device)  # noqa: E731
        self.k = zeros(n_block, head_dim // 16, BLOCK, 16, dtype=torch.int8)
        self.v = zeros(n_block, 4, head_dim, 16, dtype=torch.int8)
        self.k_scale, self.v_scale = (zeros(n_block, dtype=torch.float32) for _ in range(2))
        self.k_tail = zeros(2, head_dim // 8, BLOCK, 8, dtype=torch.float16)
        self.v_tail = zeros(2, 2, 4, head_dim, 8, dtype=torch.float16)
        self.n_req, self.n_kv_head, self.n_block, self.head_dim = n_req, n_kv_head, n_block, head_dim
        self.device = self.k.device
        self._index = self.device.index
        self._scale = 1.0 / math.sqrt(head_dim)
        self._lib = load()
        self._c = PdByteCache(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                              self.k_tail.data_ptr(), self.v_tail.data_ptr(), n_req, n_kv_head, head_dim, n_block)
        self._p = C.byref(self._c)
        # (what the pointers lead to lives as long as they do, whatever becomes of the attributes)
        self._held = (self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail)

    # -- in and out, in the plain order of tokens and dims -------------------------
    def to_tensors(self):
        """What the cache holds in plain order: k int8 [req][head][block][64][dim], v int8 [req][head][block][dim][64], k_scale,
        v_scale, k_tail half [req][head][2][64][dim], v_tail half [req][head][2][dim][64] (copies)."""
        r, h, n, d = self.n_req, self.n_kv_head, self.n_block, self.head_dim
        return {"k": self.k.transpose(3, 4).reshape(r, h, n, BLOCK, d),
                "v": self.v.view(r, h, n, 4, d, 4, 4).permute(0, 1, 2, 4, 5, 3, 6).reshape(r, h, n, d, BLOCK),
                "k_scale": self.k_scale.clone(), "v_scale": self.v_scale.clone(),
                "k_tail": self.k_tail.transpose(3, 4).reshape(r, h, 2, BLOCK, d),
                "v_tail": self.v_tail.view(r, h, 2, 2, 4, d, 2, 4).permute(0, 1, 2, 5, 3, 6, 4, 7).reshape(r, h, 2, d, BLOCK)}

    @classmethod
    def from_tensors(cls, k, v, k_scale, v_scale, k_tail, v_tail):
        """A cache that holds what these tensors hold (the ones of to_tensors, on its device; copied).  Codes are within
        [-127, 127], and 0 where the scale is 0; scales are 0 or within [2^-32, 2^32]."""
        _require(k.dim() == 5 and k.shape[3] == BLOCK, "k must be [req][head][block][%d][dim], not %s", BLOCK, tuple(k.shape))
        r, h, n, _, d = k.shape
        for name, t, shape, dtype in (("k", k, k.shape, torch.int8), ("v", v, (r, h, n, d, BLOCK), torch.int8),
                                      ("k_scale", k_scale, (r, h, n), torch.float32), ("v_scale", v_scale, (r, h, n), torch.float32),
                                      ("k_tail", k_tail, (r, h, 2, BLOCK, d), torch.float16),
                                      ("v_tail", v_tail, (r, h, 2, d, BLOCK), torch.float16)):
            _require(t.shape == tuple(shape) and t.dtype == dtype and t.device == k.device, "%s must be %s %s on %s, not %s %s on %s",
                     name, dtype, tuple(shape), k.device, t.dtype, tuple(t.shape), t.device)
        self = cls(r, h, d, n * BLOCK, device=k.device)
        self.k.copy_(k.reshape(r, h, n, BLOCK, d // 16, 16).transpose(3, 4))
        self.v.view(r, h, n, 4, d, 4, 4).copy_(v.reshape(r, h, n, d, 4, 4, 4).permute(0, 1, 2, 5, 3, 4, 6))
        self.k_scale.copy_(k_scale)
        self.v_scale.copy_(v_scale)
        self.k_tail.copy_(k_tail.reshape(r, h, 2, BLOCK, d // 8, 8).transpose(3, 4))
        self.v_tail.view(r, h, 2, 2, 4, d, 2, 4).copy_(v_tail.reshape(r, h, 2, d, 2, 2, 4, 4).permute(0, 1, 2, 4, 6, 3, 5, 7))
        return self

    # -- what every call checks --------------------------------------------------
    # (a call is bound by the host: it costs 6-8 us, of which these are two)
    def _data(self, name, t, shape):
        """Pointer, strides and type of a tensor [req][token or row][head][dim] whose dims lie together."""
        kind = _TYPES.get(t.dtype)
        if kind is None or t.shape != shape or t.device != self.device:
            raise PdError(f"{name} must be float32, bfloat16 or float16 {shape} on {self.device}, not {t.dtype} "
                          f"{tuple(t.shape)} on {t.device}")
        request, row, head, one = t.stride()
        if one != 1:
            raise PdError(f"the dims of {name} must lie together")
        return t.data_ptr(), _I64x3(request, row, head), kind

    def _ints(self, name, t, shape, dtype=torch.int32):
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype or t.device != self.device or not t.is_contiguous():
            raise PdError(f"{name} must be contiguous {dtype} {shape} on {self.device}, not {t.dtype} {tuple(t.shape)} on "
                          f"{t.device}")
        return t.data_ptr()

    def _call(self, function, *args):
        index = self._index
        if index == _current_device():
            rc = function(self._p, *args, _raw_stream(index))
        else:
            with torch.cuda.device(index):
                rc = function(self._p, *args, _raw_stream(index))
        if rc:
            _check(rc)

    # -- the operators -----------------------------------------------------------
    def append(self, k, v, lens, counts=None):
        """Stores new tokens k, v [req][new][head][dim] (fp32, bf16 or fp16) behind those that the requests hold.

        lens: int32 [req], tokens of each request with the new ones; counts: int32 [req] or None, how many are new (None: all of
        k and v; fewer: the rest is padding).  A request whose numbers do not fit is left as it is."""
        shape = k.shape
        if len(shape) != 4:
            raise PdError(f"k must be [req][new][head][dim], not {tuple(shape)}")
        n_req, n_new = self.n_req, shape[1]
        shape = (n_req, n_new, self.n_kv_head, self.head_dim)
        kp, ks, kind = self._data("k", k, shape)
        vp, vs, kind_v = self._data("v", v, shape)
        if kind != kind_v:
            raise PdError(f"k and v must have the same type, not {k.dtype} and {v.dtype}")
        self._call(self._lib.pd_byte_append, kp, vp, kind, ks, vs, n_new,
                   None if counts is None else self._ints("counts", counts, (n_req,)), self._ints("lens", lens, (n_req,)))

    def read(self, lens, n_tok, first=None, dtype=torch.float32):
        """Keys and values [req][n_tok][head][dim] of tokens first[r] .. first[r] + n_tok - 1 (int32 [req]; None: from 0) as the
        values that they stand for; zeros where a request holds none."""
        kind, n_req = _TYPES.get(dtype), self.n_req
        if n_tok < 0 or kind is None:
            raise PdError(f"n_tok must be >= 0, not {n_tok}" if n_tok < 0 else
                          f"dtype must be float32, bfloat16 or float16, not {dtype}")
        k, v = self.k_tail.new_empty((2, n_req, n_tok, self.n_kv_head, self.head_dim), dtype=dtype).unbind()
        self._call(self._lib.pd_byte_read, None if first is None else self._ints("first", first, (n_req,)), n_tok,
                   self._ints("lens", lens, (n_req,)), k.data_ptr(), v.data_ptr(), kind)
        return k, v

    def attention(self, q, lens, row_limit=None, key_tag=None, row_tag=None, scale=None, max_len=0, with_lse=False):
        """softmax(scale q k) v of query rows q [req][row][head][dim]; returns the same shape and type (and, with_lse, the
        logarithms of the sums, fp32 [req][row][head]).

        A row sees the tokens below lens[request] and, where given, below row_limit (int32 [req][row]) and with key_tag (uint16
        [req][n_block * 64]) at most row_tag (int32 [req][row]); one that sees nothing gives zeros.  head: a multiple of the
        key heads, each of which serves the query heads in turn.  scale: 1 / sqrt(dim) unless given.  max_len: a number that
        no entry of lens exceeds, if known (shorter launches)."""
        shape = q.shape
        if len(shape) != 4:
            raise PdError(f"q must be [req][row][head][dim], not {tuple(shape)}")
        n_req = self.n_req
        _, rows, heads, _ = shape
        if max_len > self.n_block * BLOCK:                # (all there is room for; the C argument has 32 bits and no checks)
            max_len = 0
        qp, qs, kind = self._data("q", q, (n_req, rows, heads, self.head_dim))
        need = self._lib.pd_byte_attention_workspace_bytes(self._p, heads, rows, max_len)
        if need == 0:
            raise PdError(f"invalid attention: {self._lib.pd_last_error().decode()}")
        out = q.new_empty(shape)
        lse = q.new_empty((n_req, rows, heads), dtype=torch.float32) if with_lse else None
        # of the caller's stream, or of the graph that captures it: never shared by two calls that may overlap
        work = q.new_empty(need, dtype=torch.uint8) if need > 16 else None
        self._call(self._lib.pd_byte_attention, qp, kind, qs, heads, rows, self._ints("lens", lens, (n_req,)),
                   None if row_limit is None else self._ints("row_limit", row_limit, (n_req, rows)),
                   None if key_tag is None else self._ints("key_tag", key_tag, (n_req, self.n_block * BLOCK), torch.uint16),
                   None if row_tag is None else self._ints("row_tag", row_tag, (n_req, rows)),
                   self._scale if scale is None else scale, max_len, out.data_ptr(),
                   None if lse is None else lse.data_ptr(), None if work is None else work.data_ptr(), need)
        return (out, lse) if with_lse else out
