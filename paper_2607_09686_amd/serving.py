"""What a decoder runs beside the MoE layer calls: a paged key/value cache with the attention that
reads it (moe_kv_append, moe_kv_attend) and the choice of the next tokens (moe_sample).

Argument marshalling only.  Every call queues its kernels on torch's current stream of the
tensors' device and returns without waiting.  Buffers that a call returns and its workspace come
from torch's allocator on that stream, so calls on several streams, and captured graphs, do not
share them.  Kernels never touch memory outside the tensors given, whatever the index tensors hold.
"""
import ctypes

from .moecache import KvBatch, KvRope, MOE_BF16, MOE_F16, MOE_F32, SampleBatch, _check, lib

# torch and its dtypes' codes: bound on first use, so that importing the package does not import torch
_torch = None
_codes = {}


def _bind():
    global _torch
    import torch
    _codes.update({torch.bfloat16: MOE_BF16, torch.float16: MOE_F16, torch.float32: MOE_F32})
    _torch = torch
    return torch


def _gpu(t, what, dtype, device):
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{what} must live on {device}, not on {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")


def _vector(t, what, dtype, n, device):
    """Pointer of a contiguous device vector of n elements."""
    _gpu(t, what, dtype, device)
    if t.shape != (n,):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {(n,)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _rows(t, what, dtype, heads, dim, n, device):
    """(pointer, stride) of token rows [n, heads, dim]; only the first dimension may have a stride."""
    _gpu(t, what, dtype, device)
    if t.requires_grad and _torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which the cache's calls do not give: detach it, or call "
                         "under torch.no_grad()")
    if t.shape != (n, heads, dim):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {(n, heads, dim)}")
    s0, s1, s2 = t.stride()
    if (heads > 1 and s1 != dim) or s2 != 1:
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    return t.data_ptr(), s0 if n > 1 else heads * dim


def _stream(index):
    """torch's current stream of a device as a hipStream_t (torch.cuda.current_stream's, without
    the objects around it: this is on the path of every decode step)."""
    return _torch._C._cuda_getCurrentRawStream(index)


def _run(index, call, *args):
    """A C entry with the device current: the null stream is the current device's."""
    if _torch._C._cuda_getDevice() == index:
        _check(call(*args))
    else:
        with _torch.cuda.device(index):
            _check(call(*args))


class KvCache:
    """Keys and values of a model's layers in fixed pages (the layout is moe_kv_batch's).

    `keys` [n_layers, n_pages, n_kv_heads, page_tokens / 16, head_dim / 8, 16, 8] and `values`
    [n_layers, n_pages, n_kv_heads, page_tokens / 16, 2, head_dim, 8] are allocated (uninitialised)
    unless given.  Which sequence holds which pages is the caller's: every call takes

      pages    int32 [n_seqs, max_pages], page ids in token order (anything for pages past the length, and
               for those that the window has passed for every new token)
      starts   int32 [n_seqs + 1], the sequences' first rows among the new tokens; rows from
               starts[n_seqs] on (a padded batch) are left alone
      lengths  int32 [n_seqs], tokens of each sequence, the new ones counted

    on the GPU; a captured graph sees their contents at replay.  `status`, an int32 tensor of one
    element, gets MOE_KV_BAD_* bits or-ed in when they are out of range.

    No call has a backward pass: rows that require a gradient are refused where gradients are recorded.

    rope_dim elements of each head turn by position * rope_theta ** (-2 i / rope_dim), or by
    rope_freqs[i], as pairs (i, i + rope_dim / 2), or (2 i, 2 i + 1) with rope_adjacent; 0: none.
    scale defaults to head_dim ** -0.5; window > 0 limits a token to that many last tokens.
    """

    def __init__(self, n_layers, n_heads, n_kv_heads, head_dim, page_tokens, n_pages, dtype=None,
                 rope_theta=10000.0, rope_dim=None, rope_adjacent=False, rope_freqs=None, scale=None,
                 window=0, device="cuda", keys=None, values=None):
        torch = _bind()
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"dtype must be torch.bfloat16 or torch.float16, got {dtype}")
        if min(n_layers, n_heads, n_kv_heads, n_pages) < 1 or n_heads % n_kv_heads:
            raise ValueError("n_layers, n_heads, n_kv_heads and n_pages must be positive, n_heads a multiple "
                             "of n_kv_heads")
        if head_dim not in (64, 128, 256):
            raise ValueError("head_dim must be 64, 128 or 256")
        if not 16 <= page_tokens <= 1024 or page_tokens & (page_tokens - 1):
            raise ValueError("page_tokens must be a power of two in [16, 1024]")
        self.n_layers, self.n_heads, self.n_kv_heads = n_layers, n_heads, n_kv_heads
        self.head_dim, self.page_tokens, self.n_pages = head_dim, page_tokens, n_pages
        self.dtype, self.window = dtype, int(window)
        self.scale = head_dim ** -0.5 if scale is None else float(scale)
        front = (n_layers, n_pages, n_kv_heads, page_tokens // 16)
        shapes = front + (head_dim // 8, 16, 8), front + (2, head_dim, 8)
        for name, t, shape in (("keys", keys, shapes[0]), ("values", values, shapes[1])):
            if t is None:
                t = torch.empty(shape, dtype=dtype, device=device)
            elif t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {dtype} of shape {shape}")
            setattr(self, "_" + name, t)  # fixed from here on: calls hold their addresses
        self.device = self.keys.device
        if self.values.device != self.device:
            raise ValueError("keys and values must live on one device")
        self.rope_dim = head_dim if rope_dim is None else int(rope_dim)
        self.rope_adjacent = bool(rope_adjacent)
        if rope_freqs is None:
            if not 0 <= self.rope_dim <= head_dim or self.rope_dim % 16:
                raise ValueError("rope_dim must be a multiple of 16 up to head_dim")
            rope_freqs = [float(rope_theta) ** (-2 * i / self.rope_dim) for i in range(self.rope_dim // 2)]
        self._rope_freqs = torch.as_tensor(rope_freqs, dtype=torch.float64).to(self.device).contiguous()
        if self.rope_freqs.shape != (self.rope_dim // 2,):
            raise ValueError(f"rope_freqs must hold {self.rope_dim // 2} frequencies")
        self._blank = None     # the batch struct's bytes up to the call's own fields, per layer
        if self.keys.is_cuda:  # made here, so that the first calls of several threads find it whole
            self._blank = [bytes(KvBatch(_codes[dtype], n_heads, n_kv_heads, head_dim, page_tokens, n_pages,
                                         0, 0, 0, 0, k.data_ptr(), v.data_ptr()))
                           for k, v in zip(self.keys, self.values)]
            self._index = self.device.index
            self._rope = KvRope(self.rope_dim, self.rope_adjacent, self.rope_freqs.data_ptr())
        self._work_bytes = {}  # a batch's counts: bytes of moe_kv_attend's workspace

    keys = property(lambda self: self._keys)
    values = property(lambda self: self._values)
    rope_freqs = property(lambda self: self._rope_freqs)

    @property
    def token_bytes(self):
        """Bytes of one token in every layer: kv_bytes_per_token of plan_percent and plan_bytes."""
        return 4 * self.n_layers * self.n_kv_heads * self.head_dim

    def _batch(self, layer, pages, starts, lengths, n_tokens, status):
        if self._blank is None:
            raise ValueError("the cache must live on the GPU")
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer {layer} outside [0, {self.n_layers})")
        i32, device = _torch.int32, self.device
        _gpu(pages, "pages", i32, device)
        if pages.dim() != 2 or not pages.is_contiguous():
            raise ValueError("pages must be a contiguous [n_seqs, max_pages] tensor")
        b = KvBatch.from_buffer_copy(self._blank[layer])
        n, b.max_pages = pages.shape
        b.n_seqs, b.n_tokens = n, n_tokens
        b.pages = pages.data_ptr()
        b.starts = _vector(starts, "starts", i32, n + 1, device)
        b.lengths = _vector(lengths, "lengths", i32, n, device)
        if status is not None:
            b.status = _vector(status, "status", i32, 1, device)
        b.hip_stream = _stream(self._index)
        return b

    def append(self, k, v, pages, starts, lengths, layer=0, q=None, q_out=None, status=None):
        """Turn k by its positions and write k and v, [tokens, n_kv_heads, head_dim] in the cache's
        dtype or float32, into their pages; with q [tokens, n_heads, head_dim] of the same dtype, also
        turn q and return it in the cache's dtype (in q_out if given, which may be q)."""
        n, kind, device, heads, dim = k.shape[0], k.dtype, self.device, self.n_heads, self.head_dim
        if kind != self.dtype and kind != _torch.float32:
            raise TypeError(f"k must be {self.dtype} or torch.float32, got {kind}")
        kp, ks = _rows(k, "k", kind, self.n_kv_heads, dim, n, device)
        vp, vs = _rows(v, "v", kind, self.n_kv_heads, dim, n, device)
        qp = qs = op = os = 0
        if q is not None:
            qp, qs = _rows(q, "q", kind, heads, dim, n, device)
            if q_out is None:
                q_out = _torch.empty((n, heads, dim), dtype=self.dtype, device=device)
            op, os = _rows(q_out, "q_out", self.dtype, heads, dim, n, device)
        elif q_out is not None:
            raise ValueError("q_out without q")
        b = self._batch(layer, pages, starts, lengths, n, status)
        _run(self._index, lib().moe_kv_append, b, self._rope, _codes[kind], kp, ks, vp, vs, qp, qs, op, os)
        return q_out

    def attend(self, q, pages, starts, lengths, layer=0, out=None, status=None):
        """Attention of the new tokens' queries q [tokens, n_heads, head_dim] (turned, in the cache's
        dtype) over their sequences, whose new tokens have been appended.  Returns out, like q."""
        n, device, heads, dim = q.shape[0], self.device, self.n_heads, self.head_dim
        qp, qs = _rows(q, "q", self.dtype, heads, dim, n, device)
        if out is None:
            out = _torch.empty((n, heads, dim), dtype=self.dtype, device=device)
        op, os = _rows(out, "out", self.dtype, heads, dim, n, device)
        b = self._batch(layer, pages, starts, lengths, n, status)
        counts = n, b.n_seqs, b.max_pages  # what the workspace's size goes by
        size = self._work_bytes.get(counts)
        if size is None:
            need = ctypes.c_uint64()
            _check(lib().moe_kv_attend_workspace(b, need))
            if len(self._work_bytes) > 4096:
                self._work_bytes.clear()
            size = self._work_bytes[counts] = need.value
        work = _torch.empty(size, dtype=_torch.uint8, device=device)
        _run(self._index, lib().moe_kv_attend, b, self.window, self.scale, qp, qs, op, os, work.data_ptr(), size)
        return out


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Choose a token from each row of logits [rows, vocab] (float32, bfloat16 or float16; rows may
    have a stride) with the uniform numbers u [rows] in [0, 1): moe_sample, which defines the filters
    and their order.  temperature, top_p, min_p (float32 [rows]) and top_k (int32 [rows]) may be
    None.  Returns (tokens int32 [rows], probs float32 [rows]); neither carries a gradient."""
    torch = _torch or _bind()
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise ValueError("logits must be a tensor on the GPU")
    kind = logits.dtype
    if kind not in _codes:
        raise TypeError(f"logits must be float32, bfloat16 or float16, got {kind}")
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    dev, (n, vocab), f32 = logits.device, logits.shape, torch.float32
    b = SampleBatch(_codes[kind], n, vocab, 0, logits.data_ptr(), logits.stride(0) if n > 1 else vocab)
    if temperature is not None:
        b.temperature = _vector(temperature, "temperature", f32, n, dev)
    if top_k is not None:
        b.top_k = _vector(top_k, "top_k", torch.int32, n, dev)
    if top_p is not None:
        b.top_p = _vector(top_p, "top_p", f32, n, dev)
    if min_p is not None:
        b.min_p = _vector(min_p, "min_p", f32, n, dev)
    b.u = _vector(u, "u", f32, n, dev)
    b.hip_stream = _stream(dev.index)
    size = _sample_bytes.get((n, vocab))
    if size is None:
        need = ctypes.c_uint64()
        _check(lib().moe_sample_workspace(b, need))
        if len(_sample_bytes) > 4096:
            _sample_bytes.clear()
        size = _sample_bytes[n, vocab] = need.value
    tokens = torch.empty(n, dtype=torch.int32, device=dev)
    probs = torch.empty(n, dtype=f32, device=dev)
    work = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
    _run(dev.index, lib().moe_sample, b, tokens.data_ptr(), probs.data_ptr(), work.data_ptr() if size else None, size)
    return tokens, probs


_sample_bytes = {}  # (rows, vocab): bytes of moe_sample's workspace
