"""Keys and values of many sequences in pages: a holder of the tensors, and the calls of include/kvp.h that serve many sequences at
once with torch tensors as their arguments.  Marshalling only, as in binding.py; calls on torch's current stream and device go
through csrc/fast_calls.cpp, and what it does not take through Python, which says what is wrong."""
import contextlib
import ctypes

from .binding import _entries, _fast_call
from .binding import KVP_EINVAL, KVP_PAGE_BF16, KVP_PAGE_E4M3, KvpError, KvpPages, KvpPrompts, KvpRows, lib


def _need(ok, what):
    if not ok:
        raise KvpError(KVP_EINVAL, what)


_prompt = None


class _On:
    """The device and stream of a call: torch's current stream of the tensors' device, or the caller's."""

    def __init__(self, device, stream):
        import torch
        self.index = device.index
        self.handle = torch._C._cuda_getCurrentRawStream(self.index)
        self.others = None
        if stream is not None:
            handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
            if handle != self.handle:
                self.handle, self.others = handle, torch.cuda.ExternalStream(handle, device=device)
        self.away = torch._C._cuda_getDevice() != self.index

    def __enter__(self):
        """What is allocated inside belongs to the call's stream."""
        import torch
        self.stack = None
        if self.away or self.others is not None:
            self.stack = contextlib.ExitStack()
            if self.away:
                self.stack.enter_context(torch.cuda.device(self.index))
            if self.others is not None:
                self.stack.enter_context(torch.cuda.stream(self.others))
        return self.handle

    def __exit__(self, *of):
        if self.stack is not None:
            self.stack.__exit__(*of)


def _numbers(t, shape, device, what):
    """(address, token stride, head stride) of bf16 rows [tokens, heads, d]."""
    import torch
    _need(t.dtype is torch.bfloat16 and t.device == device and t.shape == shape, what)
    token, head, one = t.stride()
    _need(one == 1, what)
    return t.data_ptr(), token if shape[0] > 1 else 0, head if shape[1] > 1 else 0


def _whole(t, shape, device, what):
    """Address of contiguous int32 numbers."""
    import torch
    _need(t.dtype is torch.int32 and t.device == device and t.shape == shape and t.is_contiguous(), what)
    return t.data_ptr()


def prompt_attention(q, k, v, seq_begin, out=None, softmax_scale=0.0, stream=None):
    """Causal attention inside each of the prompts whose rows are seq_begin[s] .. seq_begin[s + 1] - 1 of q [n_tokens, n_q_heads, d] and
    of k and v [n_tokens, n_kv_heads, d], any strides but the last (kvp_prompt_attention).  Rows behind the last prompt are left as they
    were in `out`; without one given they hold whatever was there, and the call takes the host 12 us, with one 4.5."""
    import torch
    global _prompt
    what, device = "prompt_attention: ", q.device
    if stream is None and out is not None and device.index is not None and torch._C._cuda_getDevice() == device.index:
        if _prompt is None:
            _prompt = _fast_call("prompt")
        rc = _prompt(_entries.kvp_prompt_attention, device.index, torch._C._cuda_getCurrentRawStream(device.index), q, k, v, seq_begin, out, softmax_scale)
        if rc == 0:
            return out
        if rc is not None:
            raise KvpError(rc, "kvp_prompt_attention")
    _need(q.dim() == 3 and k.dim() == 3 and device.type == "cuda" and device.index is not None, what + "q and k")
    (n_tokens, n_q_heads, d), n_kv_heads, n_seqs = q.shape, k.shape[1], seq_begin.numel() - 1
    at = [_numbers(q, (n_tokens, n_q_heads, d), device, what + "q")]
    at += [_numbers(t, (n_tokens, n_kv_heads, d), device, what + "k and v") for t in (k, v)]
    begin = _whole(seq_begin, (n_seqs + 1,), device, what + "seq_begin")
    with _On(device, stream) as handle:
        if out is None:
            out = torch.empty((n_tokens, n_q_heads, d), dtype=torch.bfloat16, device=device)
        at.append(_numbers(out, (n_tokens, n_q_heads, d), device, what + "out"))
        prompts = KvpPrompts(*(x[0] for x in at), begin, *(s for x in at for s in x[1:]), n_tokens, n_seqs, n_q_heads, n_kv_heads, d, softmax_scale)
        rc = lib().kvp_prompt_attention(ctypes.byref(prompts), handle)
    if rc:
        raise KvpError(rc, "kvp_prompt_attention")
    return out


class Pages:
    """Pages of one layer over the caller's tensors, [n_pages, n_kv_heads, page_size, head_dim]: `k` and `v` of bf16, or of e4m3
    (torch.float8_e4m3fn) with exponents `k_exp` and `v_exp`, uint8 [n_pages, n_kv_heads, page_size].  The tensors are kept, and cannot be
    exchanged; a call after one of them has been given other memory (resize_, set_) is refused."""

    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_exp = property(lambda self: self._tensors[2])
    v_exp = property(lambda self: self._tensors[3])
    device = property(lambda self: self._device)
    n_pages = property(lambda self: self._shape[0])
    n_kv_heads = property(lambda self: self._shape[1])
    page_size = property(lambda self: self._shape[2])
    head_dim = property(lambda self: self._shape[3])
    of = property(lambda self: KvpPages.from_buffer_copy(self._of), doc="For the calls of include/kvp.h, a copy.")

    def __init__(self, k, v, k_exp=None, v_exp=None):
        import torch
        e4m3 = k.dtype is torch.float8_e4m3fn
        _need(k.dim() == 4 and (e4m3 or k.dtype is torch.bfloat16), "Pages: k")
        _need(v.shape == k.shape and v.dtype is k.dtype and v.device == k.device, "Pages: v")
        _need(k.is_contiguous() and v.is_contiguous(), "Pages: contiguous k and v")
        _need(k.device.type == "cuda" and k.device.index is not None, "Pages: on a GPU")
        for t in (k_exp, v_exp):
            _need((t is not None) == e4m3, "Pages: exponents belong to e4m3")
            if t is not None:
                _need(t.shape == k.shape[:3] and t.dtype is torch.uint8 and t.device == k.device and t.is_contiguous(), "Pages: exponents")
        self._tensors, self._device, self._shape = (k, v, k_exp, v_exp), k.device, tuple(k.shape)
        self._of = KvpPages(k.data_ptr(), v.data_ptr(), k_exp.data_ptr() if e4m3 else None, v_exp.data_ptr() if e4m3 else None,
                            KVP_PAGE_E4M3 if e4m3 else KVP_PAGE_BF16, *k.shape)
        self._ref, self._lib = ctypes.byref(self._of), lib()
        # what every call needs, looked up once (rows of a few sequences take the GPU 2.6 us; through Python alone a call took the host 8)
        native = _fast_call("page_rows"), _fast_call("paged_decode")
        device, stream, index = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, k.device.index
        at, heads, dim, work = (ctypes.addressof(self._of), *self._tensors), k.shape[1], k.shape[3], {}
        rows, decode, write_entry, read_entry, decode_entry = *native, _entries.kvp_page_write, _entries.kvp_page_read, _entries.kvp_paged_decode
        self._work = work

        def native_write(k, v, seq_begin, table, first):
            if device() == index:
                return rows(write_entry, at, heads, dim, index, stream(index), k, v, seq_begin, table, first)

        def native_read(k, v, seq_begin, table, first):
            if device() == index:
                return rows(read_entry, at, heads, dim, index, stream(index), k, v, seq_begin, table, first)

        def native_decode(q, n_q_heads, table, lengths, out, workspace, softmax_scale):
            if device() == index:
                return decode(decode_entry, at, n_q_heads, dim, index, stream(index), q, table, lengths, out, workspace, softmax_scale)

        self._native_write, self._native_read, self._native_decode = native_write, native_read, native_decode

    @classmethod
    def empty(cls, n_pages, n_kv_heads, head_dim, page_size=64, e4m3=False, device="cuda:0"):
        """New tensors, not filled."""
        import torch
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=device)
        if not e4m3:
            return cls(new(shape, torch.bfloat16), new(shape, torch.bfloat16))
        return cls(new(shape, torch.float8_e4m3fn), new(shape, torch.float8_e4m3fn), new(shape[:3], torch.uint8), new(shape[:3], torch.uint8))

    def _need_memory(self):
        """The tensors' memory is where it was when its addresses were taken.  (The native calls look for themselves.)"""
        of = self._of
        for t, at in zip(self._tensors, (of.k, of.v, of.k_exp, of.v_exp)):
            _need(t is None or t.data_ptr() == at, "Pages: a tensor has other memory than it had")

    def _rows(self, call, k, v, seq_begin, table, first, stream):
        self._need_memory()
        n_tokens, n_seqs, device = k.shape[0], seq_begin.numel() - 1, self.device
        what = "Pages.%s: " % call
        shape = (n_tokens, self.n_kv_heads, self.head_dim)
        k_at, k_token, k_head = _numbers(k, shape, device, what + "k")
        v_at, v_token, v_head = _numbers(v, shape, device, what + "v")
        _need(table.dim() == 2, what + "table")
        rows = KvpRows(k_at, v_at, k_token, k_head, v_token, v_head, n_tokens)
        args = (self._ref, ctypes.byref(rows), _whole(seq_begin, (n_seqs + 1,), device, what + "seq_begin"),
                _whole(table, (n_seqs, table.shape[1]), device, what + "table"), table.shape[1],
                None if first is None else _whole(first, (n_seqs,), device, what + "first"), n_seqs)
        with _On(device, stream) as handle:
            rc = getattr(self._lib, "kvp_page_" + call)(*args, handle)
        if rc:
            raise KvpError(rc, "kvp_page_" + call)

    def write(self, k, v, seq_begin, table, first=None, stream=None):
        """Rows seq_begin[s] .. seq_begin[s + 1] - 1 of k and v [n_tokens, n_kv_heads, head_dim] (any strides but the last) become
        tokens first[s], first[s] + 1, ... of sequence s, whose pages are table[s] (kvp_page_write)."""
        rc = self._native_write(k, v, seq_begin, table, first) if stream is None else None
        if rc is None:
            self._rows("write", k, v, seq_begin, table, first, stream)
        elif rc:
            raise KvpError(rc, "kvp_page_write")

    def read(self, k, v, seq_begin, table, first=None, stream=None):
        """The way back, into k and v (kvp_page_read)."""
        rc = self._native_read(k, v, seq_begin, table, first) if stream is None else None
        if rc is None:
            self._rows("read", k, v, seq_begin, table, first, stream)
        elif rc:
            raise KvpError(rc, "kvp_page_read")

    def _workspace_bytes(self, n_q_heads):
        nbytes = self._work.get(n_q_heads)
        if nbytes is None:
            nbytes = self._work[n_q_heads] = self._lib.kvp_paged_decode_bytes(self._ref, n_q_heads)
        _need(nbytes > 0, "Pages.decode: n_q_heads")
        return nbytes

    def workspace(self, n_q_heads):
        """Room for the partial results of a decode step with this many query heads; steps that may overlap need one each."""
        import torch
        return torch.empty(self._workspace_bytes(n_q_heads), dtype=torch.uint8, device=self.device)

    def decode(self, q, table, lengths, out=None, softmax_scale=0.0, workspace=None, stream=None):
        """One token of every sequence: q [n_seqs, n_q_heads, head_dim] over tokens 0 .. lengths[s] - 1 of the pages table[s]
        (kvp_paged_decode).  Without a workspace one is allocated for the call.  With `out` given the call takes the host 5 us, without it 12.  A table
        that is no wider than the longest sequence needs is faster: short sequences then take one launch."""
        import torch
        if stream is None and out is not None:
            n_q_heads = q.shape[-2] if q.dim() > 1 else 0
            room = workspace if workspace is not None else self._work.get(n_q_heads) or self._workspace_bytes(n_q_heads)
            rc = self._native_decode(q, n_q_heads, table, lengths, out, room, softmax_scale)
            if rc == 0:
                return out
            if rc is not None:
                raise KvpError(rc, "kvp_paged_decode")
        self._need_memory()
        n_seqs, device = lengths.numel(), self.device
        _need(q.dim() == 3 and table.dim() == 2, "Pages.decode: q and table")
        n_q_heads, what = q.shape[1], "Pages.decode: "
        shape = (n_seqs, n_q_heads, self.head_dim)
        q_at, q_token, q_head = _numbers(q, shape, device, what + "q")
        table_at = _whole(table, (n_seqs, table.shape[1]), device, what + "table")
        lengths_at = _whole(lengths, (n_seqs,), device, what + "lengths")
        with _On(device, stream) as handle:
            if out is None:
                out = torch.empty(shape, dtype=torch.bfloat16, device=device)
            else:
                _need(out.dtype is torch.bfloat16 and out.device == device and out.shape == shape and out.is_contiguous(), what + "out")
            if workspace is None:
                workspace = self.workspace(n_q_heads)
            _need(workspace.device == device and workspace.is_contiguous(), what + "workspace")
            rc = self._lib.kvp_paged_decode(self._ref, q_at, q_token, q_head, n_q_heads, table_at, table.shape[1], lengths_at, n_seqs,
                                            softmax_scale, out.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(), handle)
        if rc:
            raise KvpError(rc, "kvp_paged_decode")
        return out
