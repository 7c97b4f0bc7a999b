"""Convenience layer for PyTorch callers: allocates the output and the workspace with
torch (plumbing) and calls the C-ABI entry points.  No arithmetic happens here."""
from __future__ import annotations

import ctypes
import threading

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as B

_TORCH_IN = {"i8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}


class Workspace:
    """Device workspace for the cross-tile carry scan, cleared once at creation."""

    def __init__(self, rows: int, cols: int, dtype: str = "i8", s: int = 16, device="cuda"):
        self.bytes = B.tcu_scan_workspace_bytes(rows, cols, B.DTYPES[dtype], s)
        self.buf = torch.empty(self.bytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = self.buf.data_ptr() + off
        B.check(B.tcu_scan_workspace_init(self.ptr, self.bytes, torch.cuda.current_stream().cuda_stream))

    def status(self) -> int:
        return B.tcu_scan_device_status(self.ptr, torch.cuda.current_stream().cuda_stream)


def dtype_name(t: torch.Tensor) -> str:
    for k, v in _TORCH_IN.items():
        if t.dtype == v:
            return k
    raise TypeError(f"unsupported input dtype {t.dtype}")


def scan(x: torch.Tensor, s: int = 16, exclusive: bool = False, out: torch.Tensor = None,
         ws: Workspace = None) -> torch.Tensor:
    """Scan a contiguous 1-D CUDA tensor (or the rows of a 2-D one); returns int32 / fp32."""
    assert x.is_cuda and x.is_contiguous()
    dn = dtype_name(x)
    rows, cols = (1, x.numel()) if x.dim() == 1 else (x.shape[0], x.shape[1])
    if out is None:
        out = torch.empty(x.shape, dtype=torch.int32 if dn == "i8" else torch.float32, device=x.device)
    if ws is None:
        ws = Workspace(rows, cols, dn, s, x.device)
    stream = torch.cuda.current_stream().cuda_stream
    if x.dim() == 1:
        fn = B.tcu_scan_exclusive if exclusive else B.tcu_scan_inclusive
        B.check(fn(x, out, cols, B.DTYPES[dn], s, ws.ptr, ws.bytes, stream))
    else:
        B.check(B.tcu_scan_batched(x, out, rows, cols, B.DTYPES[dn], s, int(exclusive), ws.ptr, ws.bytes, stream))
    return out


def segmented_scan(x: torch.Tensor, offsets: torch.Tensor, s: int = 16, exclusive: bool = False,
                   out: torch.Tensor = None) -> torch.Tensor:
    """Scan every segment x[offsets[k]:offsets[k+1]] of a contiguous 1-D CUDA tensor on its own.  `offsets` is an
    int64 CUDA tensor, non-decreasing, from 0 to len(x)."""
    assert x.is_cuda and x.is_contiguous() and x.dim() == 1
    assert offsets.is_cuda and offsets.dtype == torch.int64 and offsets.is_contiguous() and offsets.numel() >= 1
    dn = dtype_name(x)
    n = x.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.int32 if dn == "i8" else torch.float32, device=x.device)
    ws_bytes = B.tcu_scan_segmented_workspace_bytes(n, B.DTYPES[dn], s)
    buf = torch.zeros(ws_bytes + 256, dtype=torch.uint8, device=x.device)
    ptr = buf.data_ptr() + (-buf.data_ptr()) % 256
    stream = torch.cuda.current_stream().cuda_stream
    B.check(B.tcu_scan_segmented(x, out, n, offsets, offsets.numel() - 1, B.DTYPES[dn], s, int(exclusive), ptr, ws_bytes, stream))
    B.check(B.tcu_scan_device_status(ptr, stream))
    return out


# ------------------------------------------------------------------------------------------------ language-model operators
_FLOAT = {torch.float32: B.TCU_F32, torch.float16: B.TCU_F16, torch.bfloat16: B.TCU_BF16}
# the handle alone: a torch.cuda.Stream around it costs 3 us, a third of a small call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

class _Status:
    """Where the linear-attention kernels of a device record a wait that ran out: a workspace in page-locked host memory, cleared by the
    host (a captured call leaves no clearing in its graph) and read by it without waiting for anything."""

    def __init__(self, index: int):
        size = B.tcu_linattn_workspace_bytes()
        self.buffer = torch.zeros(size + 256, dtype=torch.uint8, pin_memory=True)
        self.ptr = self.buffer.data_ptr() + (-self.buffer.data_ptr()) % 256
        self.error = ctypes.c_uint32.from_address(self.ptr + 8)          # the third word
        self.multiprocessors = torch.cuda.get_device_properties(index).multi_processor_count


_status = {}          # device index -> _Status
_status_lock = threading.Lock()


def _stream(device: torch.device) -> int:
    """The current stream of `device`, which has to be the current device (launches go there)."""
    if device.type != "cuda":
        raise ValueError(f"a CUDA tensor is needed, not one on {device}")
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    return _raw_stream(device.index)


def _status_of(index: int) -> _Status:
    held = _status.get(index)
    if held is None:
        with _status_lock:                       # (kernels write to it: no thread may drop another's)
            held = _status.get(index) or _status.setdefault(index, _Status(index))
    if held.error.value:
        held.error.value = 0
        raise RuntimeError(f"an earlier linear-attention call on cuda:{index} gave up a wait: its outputs are not valid")
    return held


def linear_attention_status(device=None) -> int:
    """Waits for the current stream of `device` (an index, "cuda" or "cuda:1"; the current device by default); 0, or
    TCU_ERR_TIMEOUT if a linear-attention call on it gave up a wait (its outputs are then not valid).  Whoever learns of it
    first clears it: this function, or the next linear-attention call on the device, which raises."""
    index = None
    if device is not None:
        device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if device.type != "cuda":
            raise ValueError(f"a CUDA device is needed, not {device}")
        index = device.index
    if index is None:
        index = torch.cuda.current_device()
    if index not in _status:
        return B.TCU_OK
    torch.cuda.current_stream(index).synchronize()
    gave_up = _status[index].error.value != 0
    _status[index].error.value = 0
    return B.TCU_ERR_TIMEOUT if gave_up else B.TCU_OK


def _written(x: torch.Tensor) -> None:
    """Tells autograd that a kernel has written to x: a backward pass that has saved x then raises instead of using what it holds now."""
    if not x.is_inference():                                # (which have no version)
        torch.autograd.graph.increment_version(x)


def _not_recorded(**arrays) -> None:
    for name, x in arrays.items():
        if x.requires_grad:
            raise RuntimeError(f"{name} requires a gradient, and this call has none: make it under torch.no_grad()")


def _no_tangents(**arrays) -> None:
    """The kernels see values alone: a tangent that one of the arrays carries would be lost."""
    for name, x in arrays.items():
        if x is not None and forward_ad.unpack_dual(x).tangent is not None:
            raise NotImplementedError(f"{name} carries a tangent: forward-mode derivatives are not computed here")


def _refuse(dtype: torch.dtype, device: torch.device, **others) -> None:
    """Says which of the arrays is not like the first one."""
    for name, x in others.items():
        if x.dtype != dtype:
            raise TypeError(f"{name} is {x.dtype}, the first argument {dtype}")
        if x.device != device:
            raise ValueError(f"{name} is on {x.device}, the first argument on {device}")


def _tokens(x: torch.Tensor):
    """An array (b, t, h, d), or packed (t, h, d), as the library takes it - features contiguous, pointer and strides multiples
    of 16 bytes - and its description (pointer, batch, token, head strides; an extent of one has stride 0).  An array that is
    not like that is copied into one that is."""
    if x.dim() == 4:
        b, t, h, d = x.shape
        sb, st, sh, sd = x.stride()
    else:
        b, (t, h, d) = 1, x.shape
        sb, (st, sh, sd) = 0, x.stride()
    if b == 1:
        sb = 0
    if t == 1:
        st = 0
    if h == 1:
        sh = 0
    ptr = x.data_ptr()
    if (sd != 1 and d > 1) or (ptr | 2 * (sb | st | sh)) & 15 or (st == 0 and t > 1):
        y = _like(x, d)
        y.copy_(x)
        return _tokens(y)
    return x, (ptr, sb, st, sh)


def _like(x: torch.Tensor, d: int) -> torch.Tensor:
    """An empty (..., d) array with the leading shape of x whose rows start on 16-byte boundaries."""
    if d % 8 == 0:
        return x.new_empty((*x.shape[:-1], d))
    return x.new_empty((*x.shape[:-1], d + (-d) % 8))[..., :d]


def _check_decay(log_decay, heads, device) -> None:
    if log_decay.dtype != torch.float32 or log_decay.shape != (heads,) or log_decay.device != device or not log_decay.is_contiguous():
        raise ValueError("log_decay: a contiguous float32 tensor of one value for each head, on the device of q")


class _Mix:
    """Checked and described arguments of one linear-attention call."""

    __slots__ = ("head", "decay", "offsets", "state_shape", "log_decay", "dk", "dv", "stream", "status")

    def __init__(self, q, k, v, log_decay, scale, offsets, **states):
        dtype, device, shape = q.dtype, q.device, q.shape
        if k.dtype != dtype or v.dtype != dtype or k.device != device or v.device != device:
            _refuse(dtype, device, k=k, v=v)
        if dtype not in (torch.float16, torch.bfloat16):
            raise TypeError(f"linear attention takes float16 or bfloat16, not {dtype}")
        packed = offsets is not None
        if len(shape) != (3 if packed else 4):
            raise ValueError("q is (batch, tokens, heads, dk), or (tokens, heads, dk) with offsets")
        if k.shape != shape or v.shape[:-1] != shape[:-1]:
            raise ValueError(f"shapes do not go together: q {tuple(shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
        tokens, heads, self.dk = shape[-3:]
        self.dv = v.shape[-1]
        if packed:
            if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous() or offsets.device != device:
                raise ValueError("offsets: a contiguous int64 tensor of batch + 1 values on the device of q")
            batch = offsets.numel() - 1
        else:
            batch = shape[0]
        _check_decay(log_decay, heads, device)
        self.state_shape = (batch, heads, self.dk, self.dv)
        for name, s in states.items():
            if s is not None and (s.shape != self.state_shape or s.dtype != torch.float32 or not s.is_contiguous() or s.device != device):
                raise ValueError(f"{name}: a contiguous float32 tensor of shape {self.state_shape} on the device of q")
        self.head = (_FLOAT[dtype], batch, tokens, heads, self.dk, self.dv, self.dk ** -0.5 if scale is None else float(scale), log_decay.data_ptr())
        self.offsets = offsets.data_ptr() if packed else 0
        self.log_decay = log_decay
        self.stream = _stream(device)
        self.status = _status_of(device.index)

    def new_state(self):
        return self.log_decay.new_empty(self.state_shape)

    def call(self, fn, backward, q, k, v, o=B.NO_TOKENS, **more):
        args = B.tcu_linattn_args(*self.head, q, k, v, o, d_offsets=self.offsets, **more)
        if self.head[1] * self.head[3] * (3 if backward else 1) > self.status.multiprocessors:
            size = B.tcu_linattn_scratch_bytes(args, backward)
            if size:
                scratch = self.log_decay.new_empty((size + 3) // 4)
                args = B.tcu_linattn_with_scratch(args, scratch.data_ptr(), size)
        B.check(fn(args, self.status.ptr, 256, self.stream))


def _ptr(x) -> int:
    return 0 if x is None else x.data_ptr()


def _out(x: torch.Tensor) -> torch.Tensor:
    return x if x.shape[-1] % 8 == 0 else x.contiguous()


def _attention_forward(q, k, v, log_decay, scale, initial_state, offsets, output_final_state):
    m = _Mix(q, k, v, log_decay, scale, offsets, initial_state=initial_state)
    last = m.new_state() if output_final_state else None
    o = _like(v, m.dv)
    (q, qv), (k, kv), (v, vv), (_, ov) = _tokens(q), _tokens(k), _tokens(v), _tokens(o)
    m.call(B.tcu_linattn_forward, 0, qv, kv, vv, ov, d_state_in=_ptr(initial_state), d_state_out=_ptr(last))
    return _out(o), last


def linear_attention_backward(d_o, q, k, v, log_decay, scale=None, initial_state=None, offsets=None, d_final_state=None):
    """Gradients of :func:`linear_attention` with respect to q, k, v and the initial state (None without one), from the
    gradient of its output and, where it has one, of the final state."""
    if forward_ad._current_level >= 0:
        _no_tangents(d_o=d_o, q=q, k=k, v=v, log_decay=log_decay, initial_state=initial_state, d_final_state=d_final_state)
    m = _Mix(q, k, v, log_decay, scale, offsets, initial_state=initial_state, d_final_state=d_final_state)
    if d_o.dtype != q.dtype or d_o.device != q.device:
        _refuse(q.dtype, q.device, d_o=d_o)
    if d_o.shape != v.shape:
        raise ValueError(f"d_o is {tuple(d_o.shape)}, v {tuple(v.shape)}")
    d_first = m.new_state() if initial_state is not None else None
    d_q, d_k, d_v = _like(q, m.dk), _like(k, m.dk), _like(v, m.dv)
    (q, qv), (k, kv), (v, vv), (d_o, ov) = _tokens(q), _tokens(k), _tokens(v), _tokens(d_o)
    m.call(B.tcu_linattn_backward, 1, qv, kv, vv, d_o=ov, d_q=_tokens(d_q)[1], d_k=_tokens(d_k)[1], d_v=_tokens(d_v)[1], d_state_in=_ptr(initial_state),
           d_dstate_out=_ptr(d_final_state), d_dstate_in=_ptr(d_first))
    return _out(d_q), _out(d_k), _out(d_v), d_first


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, scale, initial_state, offsets, output_final_state):
        ctx.save_for_backward(q, k, v, log_decay, initial_state, offsets)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return _attention_forward(q, k, v, log_decay, scale, initial_state, offsets, output_final_state)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o, d_last):
        q, k, v, log_decay, initial_state, offsets = ctx.saved_tensors
        d_o = torch.zeros_like(v) if d_o is None else d_o
        d_last = None if d_last is None else d_last.contiguous()
        d_q, d_k, d_v, d_first = linear_attention_backward(d_o, q, k, v, log_decay, ctx.scale, initial_state, offsets, d_last)
        return d_q, d_k, d_v, None, None, d_first, None, None


def linear_attention(q, k, v, log_decay, scale=None, initial_state=None, offsets=None, output_final_state=False):
    """Causal linear attention with a decay for each head: S_t = a S_{t-1} + k_t v_t^T, o_t = scale * S_t^T q_t with
    a = exp(log_decay[head]).  Returns (o, final state), the state None unless asked for; differentiable, once, in q, k, v
    and the initial state.

    q, k (batch, tokens, heads, dk) and v (batch, tokens, heads, dv), float16 or bfloat16, any strides (dk, dv at most 128);
    or packed (tokens, heads, d) with `offsets`, an int64 tensor of batch + 1 values on the GPU: sequence b is
    [offsets[b], offsets[b + 1]).  log_decay (heads,) float32, at most 0, a constant of the model (no gradient); scale: dk ** -0.5
    by default; states (batch, heads, dk, dv) float32."""
    if forward_ad._current_level >= 0 or (torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or
                                                                       (initial_state is not None and initial_state.requires_grad))):
        return _LinearAttention.apply(q, k, v, log_decay, scale, initial_state, offsets, output_final_state)
    return _attention_forward(q, k, v, log_decay, scale, initial_state, offsets, output_final_state)


def linear_attention_step(q, k, v, log_decay, state, scale=None, slots=None):
    """One token for each sequence: updates `state` in place and returns o (batch, heads, dv).  q, k (batch, heads, dk),
    v (batch, heads, dv); state (pool, heads, dk, dv) float32; slots: None (sequence b has entry b), or an int32 tensor of
    each sequence's entry, all different; an entry outside the pool marks a sequence to skip (its output is zero).
    No gradient is computed: with gradients enabled, inputs that require one are refused."""
    if forward_ad._current_level >= 0:
        _no_tangents(q=q, k=k, v=v, log_decay=log_decay, state=state)
    if torch.is_grad_enabled():
        _not_recorded(q=q, k=k, v=v, state=state)
    dtype, device, shape = q.dtype, q.device, q.shape
    if k.dtype != dtype or v.dtype != dtype or k.device != device or v.device != device:
        _refuse(dtype, device, k=k, v=v)
    if dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"linear attention takes float16 or bfloat16, not {dtype}")
    if len(shape) != 3 or k.shape != shape or v.dim() != 3 or v.shape[:2] != shape[:2]:
        raise ValueError(f"shapes do not go together: q {tuple(shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    batch, heads, dk = shape
    dv = v.shape[-1]
    pool = state.shape
    if len(pool) != 4 or pool[1:] != (heads, dk, dv) or state.dtype != torch.float32 or not state.is_contiguous() or state.device != device:
        raise ValueError(f"state: a contiguous float32 tensor of shape (pool, {heads}, {dk}, {dv}) on the device of q")
    _check_decay(log_decay, heads, device)
    if slots is not None and (slots.shape != (batch,) or slots.dtype != torch.int32 or not slots.is_contiguous() or slots.device != device):
        raise ValueError("slots: a contiguous int32 tensor of one value for each sequence, on the device of q")
    o = q.new_empty((batch, heads, dv))

    def view(x):
        sb, sh, sd = x.stride()
        if sd != 1 and x.shape[-1] > 1:
            x = x.contiguous()
            sb, sh, sd = x.stride()
        return x, (x.data_ptr(), sb, 0, sh)

    (q, qv), (k, kv), (v, vv) = view(q), view(k), view(v)
    args = B.tcu_linattn_args(_FLOAT[dtype], batch, 1, heads, dk, dv, dk ** -0.5 if scale is None else float(scale), log_decay.data_ptr(),
                              qv, kv, vv, (o.data_ptr(), heads * dv, 0, dv), d_slots=_ptr(slots), pool_slots=pool[0], d_state_out=state.data_ptr())
    B.check(B.tcu_linattn_step(args, _stream(device)))
    _written(state)
    return o


def _ids(ids: torch.Tensor, device) -> torch.Tensor:
    if ids.dtype not in (torch.int32, torch.int64) or ids.device != device:
        raise ValueError(f"ids: int32 or int64 on {device}")
    return ids.contiguous()


def embedding_backward(d_out, ids, num_rows, scale=1.0, dtype=torch.float32, out=None):
    """Gradient of :func:`embedding` with respect to its table: (num_rows, d) of `dtype` (float32, or the type of d_out), row v
    the sum of scale * d_out over the tokens with id v, zero where there is none.  With `out` the sums are added to it
    instead (rows without tokens are not touched)."""
    if forward_ad._current_level >= 0:
        _no_tangents(d_out=d_out, out=out)
    if out is not None and torch.is_grad_enabled():
        _not_recorded(out=out)
    device, kind = d_out.device, d_out.dtype
    d_out, ids = d_out.contiguous(), _ids(ids, device)
    d = d_out.shape[-1]
    if kind not in _FLOAT or d_out.shape[:-1] != ids.shape:
        raise ValueError(f"d_out {tuple(d_out.shape)} {kind} does not go with ids {tuple(ids.shape)}")
    table = out
    if out is None:
        table = torch.empty((num_rows, d), dtype=dtype, device=device)
    elif out.shape != (num_rows, d) or not out.is_contiguous() or out.device != device:
        raise ValueError(f"out: a contiguous tensor of shape ({num_rows}, {d}) on the device of d_out")
    if table.dtype != torch.float32 and table.dtype != kind:
        raise TypeError(f"the table's gradient is float32 or {kind}, not {table.dtype}")
    n = ids.numel()
    ws_bytes = B.tcu_embedding_workspace_bytes(n, num_rows, d)
    ws = ids.new_empty((ws_bytes + 7) // 8, dtype=torch.int64) if ws_bytes else None
    B.check(B.tcu_embedding_backward(d_out, _FLOAT[kind], ids, ids.element_size(), n, num_rows, d, float(scale), out is not None,
                                     table, _FLOAT[table.dtype], ws, ws_bytes, _stream(device)))
    if out is not None:
        _written(out)
    return table


def _embedding_forward(ids, table, scale):
    kind, device = table.dtype, table.device
    if table.dim() != 2 or kind not in _FLOAT:
        raise ValueError("table: (rows, d), float32, float16 or bfloat16")
    ids = _ids(ids, device)
    rows, d = table.shape
    pitch, step = table.stride()
    if (step != 1 and d > 1) or (pitch < d and rows > 1):
        table = table.contiguous()
        pitch = d
    out = table.new_empty((*ids.shape, d))
    B.check(B.tcu_embedding_forward(ids, ids.element_size(), ids.numel(), table, rows, d, max(pitch, d), _FLOAT[kind], float(scale), out, _stream(device)))
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.dtype, ctx.scale = table.shape[0], table.dtype, scale
        return _embedding_forward(ids, table, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        return None, embedding_backward(d_out, ctx.saved_tensors[0], ctx.rows, ctx.scale, ctx.dtype), None


def embedding(ids, table, scale=1.0):
    """scale * table[ids], rounded once to the table's type; an id outside the table gives a row of zeros.  ids int32 or int64
    of any shape; differentiable, once, in the table."""
    if forward_ad._current_level >= 0 or (table.requires_grad and torch.is_grad_enabled()):
        return _Embedding.apply(ids, table, scale)
    return _embedding_forward(ids, table, scale)
