"""What a decoder runs beside the MoE layer calls: a paged key/value cache with the attention that
reads it (moe_kv_append, moe_kv_attend) and the choice of the next tokens (moe_sample).

Argument marshalling only.  Every call queues its kernels on torch's current stream of the
tensors' device and returns without waiting.  Buffers that a call returns and its workspace come
from torch's allocator on that stream, so calls on several streams, and captured graphs, do not
share them.  Kernels never touch memory outside the tensors given, whatever the index tensors hold.
"""
import ctypes

from .moecache import KvBatch, KvRope, MOE_BF16, MOE_F16, MOE_F32, SampleBatch, _check, lib


def _types():
    import torch
    return {torch.bfloat16: MOE_BF16, torch.float16: MOE_F16, torch.float32: MOE_F32}


def _gpu(t, what, dtype, device):
    import torch
    if not isinstance(t, torch.Tensor):
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
    if t.dim() != 3 or t.shape[1:] != (heads, dim) or (n is not None and t.shape[0] != n):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected "
                         f"{('tokens' if n is None else n, heads, dim)}")
    if (heads > 1 and t.stride(1) != dim) or t.stride(2) != 1:
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else heads * dim


class KvCache:
    """Keys and values of a model's layers in fixed pages (the layout is moe_kv_batch's).

    `keys` [n_layers, n_pages, n_kv_heads, page_tokens / 16, head_dim / 8, 16, 8] and `values`
    [n_layers, n_pages, n_kv_heads, page_tokens / 16, 2, head_dim, 8] are allocated (uninitialised)
    unless given.  Which sequence holds which pages is the caller's: every call takes

      pages    int32 [n_seqs, max_pages], page ids in token order
      starts   int32 [n_seqs + 1], the sequences' first rows among the new tokens; rows from
               starts[n_seqs] on (a padded batch) are left alone
      lengths  int32 [n_seqs], tokens of each sequence, the new ones counted

    on the GPU; a captured graph sees their contents at replay.  `status`, an int32 tensor of one
    element, gets MOE_KV_BAD_* bits or-ed in when they are out of range.

    rope_dim elements of each head turn by position * rope_theta ** (-2 i / rope_dim), or by
    rope_freqs[i], as pairs (i, i + rope_dim / 2), or (2 i, 2 i + 1) with rope_adjacent; 0: none.
    scale defaults to head_dim ** -0.5; window > 0 limits a token to that many last tokens.
    """

    def __init__(self, n_layers, n_heads, n_kv_heads, head_dim, page_tokens, n_pages, dtype=None,
                 rope_theta=10000.0, rope_dim=None, rope_adjacent=False, rope_freqs=None, scale=None,
                 window=0, device="cuda", keys=None, values=None):
        import torch
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
            setattr(self, name, t)
        self.device = self.keys.device
        if self.values.device != self.device:
            raise ValueError("keys and values must live on one device")
        self.rope_dim = head_dim if rope_dim is None else int(rope_dim)
        self.rope_adjacent = bool(rope_adjacent)
        if rope_freqs is None:
            if not 0 <= self.rope_dim <= head_dim or self.rope_dim % 16:
                raise ValueError("rope_dim must be a multiple of 16 up to head_dim")
            rope_freqs = [float(rope_theta) ** (-2 * i / self.rope_dim) for i in range(self.rope_dim // 2)]
        self.rope_freqs = torch.as_tensor(rope_freqs, dtype=torch.float64).to(self.device).contiguous()
        if self.rope_freqs.shape != (self.rope_dim // 2,):
            raise ValueError(f"rope_freqs must hold {self.rope_dim // 2} frequencies")

    @property
    def token_bytes(self):
        """Bytes of one token in every layer: kv_bytes_per_token of plan_percent and plan_bytes."""
        return 4 * self.n_layers * self.n_kv_heads * self.head_dim

    def _batch(self, layer, pages, starts, lengths, n_tokens, status):
        import torch
        if not self.keys.is_cuda:
            raise ValueError("the cache must live on the GPU")
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer {layer} outside [0, {self.n_layers})")
        _gpu(pages, "pages", torch.int32, self.device)
        if pages.dim() != 2 or not pages.is_contiguous():
            raise ValueError("pages must be a contiguous [n_seqs, max_pages] tensor")
        n = pages.shape[0]
        return KvBatch(_types()[self.dtype], self.n_heads, self.n_kv_heads, self.head_dim, self.page_tokens,
                       self.n_pages, pages.shape[1], n, n_tokens, 0, self.keys[layer].data_ptr(),
                       self.values[layer].data_ptr(), pages.data_ptr(),
                       _vector(starts, "starts", torch.int32, n + 1, self.device),
                       _vector(lengths, "lengths", torch.int32, n, self.device),
                       None if status is None else _vector(status, "status", torch.int32, 1, self.device),
                       torch.cuda.current_stream(self.device).cuda_stream)

    def append(self, k, v, pages, starts, lengths, layer=0, q=None, q_out=None, status=None):
        """Turn k by its positions and write k and v, [tokens, n_kv_heads, head_dim] in the cache's
        dtype or float32, into their pages; with q [tokens, n_heads, head_dim] of the same dtype, also
        turn q and return it in the cache's dtype (in q_out if given, which may be q)."""
        import torch
        b = self._batch(layer, pages, starts, lengths, k.shape[0], status)
        kind = k.dtype
        if kind not in (self.dtype, torch.float32):
            raise TypeError(f"k must be {self.dtype} or torch.float32, got {kind}")
        kp, ks = _rows(k, "k", kind, self.n_kv_heads, self.head_dim, None, self.device)
        vp, vs = _rows(v, "v", kind, self.n_kv_heads, self.head_dim, k.shape[0], self.device)
        qp = qs = op = os = 0
        if q is not None:
            qp, qs = _rows(q, "q", kind, self.n_heads, self.head_dim, k.shape[0], self.device)
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
            op, os = _rows(q_out, "q_out", self.dtype, self.n_heads, self.head_dim, k.shape[0], self.device)
        elif q_out is not None:
            raise ValueError("q_out without q")
        rope = KvRope(self.rope_dim, self.rope_adjacent, self.rope_freqs.data_ptr())
        with torch.cuda.device(self.device):
            _check(lib().moe_kv_append(ctypes.byref(b), ctypes.byref(rope), _types()[kind], kp, ks, vp, vs, qp, qs,
                                       op, os))
        return q_out

    def attend(self, q, pages, starts, lengths, layer=0, out=None, status=None):
        """Attention of the new tokens' queries q [tokens, n_heads, head_dim] (turned, in the cache's
        dtype) over their sequences, whose new tokens have been appended.  Returns out, like q."""
        import torch
        qp, qs = _rows(q, "q", self.dtype, self.n_heads, self.head_dim, None, self.device)
        b = self._batch(layer, pages, starts, lengths, q.shape[0], status)
        if out is None:
            out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        op, os = _rows(out, "out", self.dtype, self.n_heads, self.head_dim, q.shape[0], self.device)
        size = ctypes.c_uint64()
        _check(lib().moe_kv_attend_workspace(ctypes.byref(b), ctypes.byref(size)))
        work = torch.empty(size.value, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            _check(lib().moe_kv_attend(ctypes.byref(b), self.window, self.scale, qp, qs, op, os, work.data_ptr(),
                                       size.value))
        return out


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Choose a token from each row of logits [rows, vocab] (float32, bfloat16 or float16; rows may
    have a stride) with the uniform numbers u [rows] in [0, 1): moe_sample, which defines the filters
    and their order.  temperature, top_p, min_p (float32 [rows]) and top_k (int32 [rows]) may be
    None.  Returns (tokens int32 [rows], probs float32 [rows])."""
    import torch
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise ValueError("logits must be a tensor on the GPU")
    if logits.dtype not in _types():
        raise TypeError(f"logits must be float32, bfloat16 or float16, got {logits.dtype}")
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    dev, (n, vocab) = logits.device, logits.shape
    row = [None if t is None else _vector(t, what, dtype, n, dev) for t, what, dtype in (
        (temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
        (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32))]
    tokens = torch.empty(n, dtype=torch.int32, device=dev)
    probs = torch.empty(n, dtype=torch.float32, device=dev)
    b = SampleBatch(_types()[logits.dtype], n, vocab, 0, logits.data_ptr(),
                    logits.stride(0) if n > 1 else vocab, *row, _vector(u, "u", torch.float32, n, dev),
                    torch.cuda.current_stream(dev).cuda_stream)
    size = ctypes.c_uint64()
    _check(lib().moe_sample_workspace(ctypes.byref(b), ctypes.byref(size)))
    work = torch.empty(size.value, dtype=torch.uint8, device=dev)
    with torch.cuda.device(dev):
        _check(lib().moe_sample(ctypes.byref(b), tokens.data_ptr(), probs.data_ptr(), work.data_ptr(), size.value))
    return tokens, probs
