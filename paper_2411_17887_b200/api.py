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


# ------------------------------------------------------------------------------------------------ gated recurrence
def _channels(x: torch.Tensor):
    """An array (b, t, d), or packed (t, d), with its channels contiguous (copied if they are not), and its description."""
    strides = x.stride()
    if strides[-1] != 1 and x.shape[-1] > 1:
        x = x.contiguous()
        strides = x.stride()
    return x, (x.data_ptr(), strides[0] if len(strides) == 3 else 0, strides[-2])


def _input_gate(name) -> int:
    kind = B.INPUT_GATES.get(name)
    if kind is None:
        raise ValueError(f"input_gate is one of {', '.join(B.INPUT_GATES)}, not {name!r}")
    return kind


class _Gated:
    """Checked and described arguments of one call of the gated recurrence over whole sequences."""

    __slots__ = ("head", "x", "offsets", "state_shape", "mark_shape", "strides", "stream")

    def __init__(self, x, gate, offsets, input_gate, **states):
        dtype, device, shape = x.dtype, x.device, x.shape
        if gate.dtype != dtype or gate.device != device:
            _refuse(dtype, device, gate=gate)
        if dtype not in _FLOAT:
            raise TypeError(f"the gated recurrence takes float32, float16 or bfloat16, not {dtype}")
        packed = offsets is not None
        if len(shape) != (2 if packed else 3):
            raise ValueError("x is (batch, tokens, channels), or (tokens, channels) with offsets")
        if gate.shape != shape:
            raise ValueError(f"shapes do not go together: x {tuple(shape)}, gate {tuple(gate.shape)}")
        if packed and (offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous() or offsets.device != device):
            raise ValueError("offsets: a contiguous int64 tensor of batch + 1 values on the device of x")
        tokens, channels = shape[-2:]
        if channels == 0:
            raise ValueError("there are no channels")
        batch = offsets.numel() - 1 if packed else shape[0]
        self.state_shape = (batch, channels)
        self.mark_shape = ((tokens if packed else batch * tokens) // 64 + batch, channels)            # (tcu_gated_marks_bytes)
        self.strides = (0 if packed else tokens * channels, channels)                                # of a fresh array
        for name, s in states.items():
            want = self.mark_shape if name == "marks" else self.state_shape
            if s is not None and (s.shape != want or s.dtype != torch.float32 or not s.is_contiguous() or s.device != device):
                raise ValueError(f"{name}: a contiguous float32 tensor of shape {want} on the device of x")
        self.head = (_FLOAT[dtype], _input_gate(input_gate), channels, batch, tokens)
        self.x = x
        self.offsets = offsets.data_ptr() if packed else 0
        self.stream = _stream(device)

    def new(self, shape):
        return torch.empty(shape, dtype=torch.float32, device=self.x.device)

    def call(self, fn, x, gate, y=B.NO_ROWS, marks=None, **more):
        B.check(fn(B.tcu_gated_args(*self.head, x, gate, y, d_offsets=self.offsets, d_marks=_ptr(marks), marks_bytes=0 if marks is None else 4 * marks.numel(), **more),
                   self.stream))


def _gated_forward(x, gate, initial_state, offsets, output_final_state, input_gate, output_marks, output=True):
    m = _Gated(x, gate, offsets, input_gate, initial_state=initial_state)
    y = _fresh(x) if output else None
    last = None
    if output_final_state:
        last = m.new(m.state_shape) if initial_state is None else torch.empty_like(initial_state)
    marks = m.new(m.mark_shape) if output_marks else None
    (x, xv), (gate, gv) = _channels(x), _channels(gate)
    m.call(B.tcu_gated_forward, xv, gv, (y.data_ptr(), *m.strides) if output else B.NO_ROWS, marks, d_state_in=_ptr(initial_state), d_state_out=_ptr(last))
    return y, last, marks


def gated_recurrence_backward(d_y, x, gate, initial_state=None, offsets=None, d_final_state=None, input_gate="complement", marks=None):
    """Gradients of :func:`gated_recurrence` with respect to x, gate and the initial state (None without one), from the gradient
    of its output and, where it has one, of the final state.  `marks`: what the forward call with these x, gate and initial state
    gave for ``output_marks=True``; without them they are computed once more."""
    if forward_ad._current_level >= 0:
        _no_tangents(d_y=d_y, x=x, gate=gate, initial_state=initial_state, d_final_state=d_final_state, marks=marks)
    if d_y.dtype != x.dtype or d_y.device != x.device:
        _refuse(x.dtype, x.device, d_y=d_y)
    if d_y.shape != x.shape:
        raise ValueError(f"d_y is {tuple(d_y.shape)}, x {tuple(x.shape)}")
    m = _Gated(x, gate, offsets, input_gate, initial_state=initial_state, d_final_state=d_final_state, marks=marks)
    if marks is None:
        marks = _gated_forward(x, gate, initial_state, offsets, False, input_gate, True, output=False)[2]
    # (nothing flows back to the rows of no sequence: the kernel sets them to zero, if there is one)
    fresh = _zeros if offsets is not None and m.state_shape[0] == 0 else _fresh
    d_x, d_gate = fresh(x), fresh(x)
    d_first = torch.empty_like(initial_state) if initial_state is not None else None
    (x, xv), (gate, gv), (d_y, yv) = _channels(x), _channels(gate), _channels(d_y)
    m.call(B.tcu_gated_backward, xv, gv, marks=marks, d_y=yv, d_x=(d_x.data_ptr(), *m.strides), d_gate=(d_gate.data_ptr(), *m.strides), d_dstate_out=_ptr(d_final_state),
           d_dstate_in=_ptr(d_first), clear_rows=int(offsets is not None))
    return d_x, d_gate, d_first


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, initial_state, offsets, output_final_state, input_gate, output_marks):
        y, last, marks = _gated_forward(x, gate, initial_state, offsets, output_final_state, input_gate, True)
        ctx.save_for_backward(x, gate, initial_state, offsets, marks)
        ctx.input_gate = input_gate
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(marks)
        return y, last, marks

    @staticmethod
    @once_differentiable
    def backward(ctx, d_y, d_last, _):
        x, gate, initial_state, offsets, marks = ctx.saved_tensors
        d_y = torch.zeros_like(x) if d_y is None else d_y
        d_last = None if d_last is None else d_last.contiguous()
        d_x, d_gate, d_first = gated_recurrence_backward(d_y, x, gate, initial_state, offsets, d_last, ctx.input_gate, marks)
        return d_x, d_gate, d_first, None, None, None, None


def gated_recurrence(x, gate, initial_state=None, offsets=None, output_final_state=False, input_gate="complement", output_marks=False):
    """Gated linear recurrence, for every channel on its own: h_t = f_t h_{t-1} + i_t x_t with f = sigmoid(gate) and i = 1 - f
    (input_gate "complement"), 1 ("one") or sqrt(1 - f^2) ("root").  Returns (h, final state), the state None unless asked for, and with
    ``output_marks=True`` (h, final state, marks), the marks for :func:`gated_recurrence_backward`; differentiable, once, in x, gate
    and the initial state.

    x, gate (batch, tokens, channels), float32, float16 or bfloat16, any strides; or packed (tokens, channels) with `offsets`, an int64
    tensor of batch + 1 values on the GPU: sequence b is [offsets[b], offsets[b + 1]), rows behind the last one are left as they
    are (of fresh memory), and their gradients are zero.  States (batch, channels) float32."""
    if forward_ad._current_level >= 0 or (torch.is_grad_enabled() and (x.requires_grad or gate.requires_grad or
                                                                       (initial_state is not None and initial_state.requires_grad))):
        y, last, marks = _GatedRecurrence.apply(x, gate, initial_state, offsets, output_final_state, input_gate, output_marks)
    else:
        y, last, marks = _gated_forward(x, gate, initial_state, offsets, output_final_state, input_gate, output_marks)
    return (y, last, marks) if output_marks else (y, last)


def gated_recurrence_step(x, gate, state, slots=None, input_gate="complement"):
    """One token for each sequence: updates `state` in place and returns h (batch, channels).  x, gate (batch, channels); state
    (pool, channels) float32; slots: None (sequence b has entry b), or an int32 tensor of each sequence's entry, all different; an entry
    outside the pool marks a sequence to skip (its output is zero).  No gradient is computed: with gradients enabled, inputs
    that require one are refused."""
    if forward_ad._current_level >= 0:
        _no_tangents(x=x, gate=gate, state=state)
    if torch.is_grad_enabled():
        _not_recorded(x=x, gate=gate, state=state)
    dtype, device, shape = x.dtype, x.device, x.shape
    if gate.dtype != dtype or gate.device != device:
        _refuse(dtype, device, gate=gate)
    if dtype not in _FLOAT:
        raise TypeError(f"the gated recurrence takes float32, float16 or bfloat16, not {dtype}")
    if len(shape) != 2 or gate.shape != shape or shape[1] == 0:
        raise ValueError(f"shapes do not go together: x {tuple(shape)}, gate {tuple(gate.shape)}")
    batch, channels = shape
    pool = state.shape
    if len(pool) != 2 or pool[1] != channels or state.dtype != torch.float32 or not state.is_contiguous() or state.device != device:
        raise ValueError(f"state: a contiguous float32 tensor of shape (pool, {channels}) on the device of x")
    if slots is not None and (slots.shape != (batch,) or slots.dtype != torch.int32 or not slots.is_contiguous() or slots.device != device):
        raise ValueError("slots: a contiguous int32 tensor of one value for each sequence, on the device of x")
    kind = _input_gate(input_gate)
    y = _fresh(x)

    def view(r):
        if channels > 1 and r.stride(1) != 1:
            r = r.contiguous()
        return r, (r.data_ptr(), r.stride(0), 0)

    (x, xv), (gate, gv) = view(x), view(gate)
    args = B.tcu_gated_args(_FLOAT[dtype], kind, channels, batch, 1, xv, gv, (y.data_ptr(), channels, 0), d_slots=_ptr(slots), pool_slots=pool[0], d_state_out=state.data_ptr())
    B.check(B.tcu_gated_step(args, _stream(device)))
    _written(state)
    return y


# ------------------------------------------------------------------------------------------------ layer norm
def _fresh(x: torch.Tensor) -> torch.Tensor:
    """An empty tensor of x's shape and type, contiguous."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _zeros(x: torch.Tensor) -> torch.Tensor:
    return torch.zeros_like(x, memory_format=torch.contiguous_format)


def _rows(x: torch.Tensor):
    """x as rows of its last axis: a tensor whose rows lie one stride apart, their number and the stride (copied if they do not)."""
    d = x.shape[-1]
    if x.dim() == 2:
        stride, step = x.stride()
        if step == 1 or d == 1:
            return x, x.shape[0], stride
    x = x.contiguous()
    return x, x.numel() // d, d


def _check_norm(x, eps, weight, bias):
    """The type of the parameters."""
    kind = None
    for name, p in (("weight", weight), ("bias", bias)):
        if p is None:
            continue
        if p.shape != x.shape[-1:] or not p.is_contiguous() or p.device != x.device:
            raise ValueError(f"{name}: a contiguous tensor of shape ({x.shape[-1]},) on the device of x")
        if p.dtype not in (torch.float32, x.dtype) or (kind is not None and p.dtype != kind):
            raise TypeError(f"{name} is {p.dtype}: float32 or the type of x, and all parameters alike")
        kind = p.dtype
    if x.dtype not in _FLOAT:
        raise TypeError(f"layer norm takes float32, float16 or bfloat16, not {x.dtype}")
    if x.dim() < 1 or x.shape[-1] == 0:
        raise ValueError(f"x is {tuple(x.shape)}: there is no last axis to normalise")
    if not 0.0 <= eps < float("inf"):
        raise ValueError(f"eps is {eps}")
    return kind or torch.float32


def _norm_forward(x, weight, bias, eps):
    kind = _check_norm(x, eps, weight, bias)
    stream = _stream(x.device)
    y = _fresh(x)
    x, rows, stride = _rows(x)
    B.check(B.tcu_layer_norm_forward(x.data_ptr(), rows, x.shape[-1], stride, _FLOAT[x.dtype], _ptr(weight), _ptr(bias), _FLOAT[kind], eps, y.data_ptr(), stream))
    return y


def layer_norm_backward(d_y, x, weight=None, eps=1e-5, params=True):
    """Gradients of :func:`layer_norm` with respect to x, weight and bias, from that of its output: (d_x, d_weight, d_bias), the
    last two of the weight's type (float32 without one), None with ``params=False``."""
    if forward_ad._current_level >= 0:
        _no_tangents(d_y=d_y, x=x, weight=weight)
    return _norm_backward(d_y, x, weight, None, eps, True, params, params)


def _norm_backward(d_y, x, weight, bias, eps, want_x, want_weight, want_bias):
    kind = _check_norm(x, eps, weight, bias)
    if d_y.dtype != x.dtype or d_y.device != x.device:
        _refuse(x.dtype, x.device, d_y=d_y)
    if d_y.shape != x.shape:
        raise ValueError(f"d_y is {tuple(d_y.shape)}, x {tuple(x.shape)}")
    d = x.shape[-1]
    d_x = _fresh(x) if want_x else None
    like = weight if weight is not None else x.new_empty(d, dtype=kind) if want_weight or want_bias else None
    d_weight = torch.empty_like(like) if want_weight else None
    d_bias = torch.empty_like(like) if want_bias else None
    x, rows, stride = _rows(x)
    d_y, _, dy_stride = _rows(d_y)
    size = B.tcu_layer_norm_workspace_bytes(rows, d) if want_weight or want_bias else 0
    ws = torch.empty(size // 4, dtype=torch.float32, device=x.device) if size else None
    B.check(B.tcu_layer_norm_backward(d_y.data_ptr(), dy_stride, x.data_ptr(), stride, rows, d, _FLOAT[x.dtype], _ptr(weight), _FLOAT[kind], eps, _ptr(d_x), _ptr(d_weight),
                                      _ptr(d_bias), _ptr(ws), size, _stream(x.device)))
    return d_x, d_weight, d_bias


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        ctx.save_for_backward(x, weight, bias)
        ctx.eps = eps
        return _norm_forward(x, weight, bias, eps)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_y):
        return (*_norm_backward(d_y, *ctx.saved_tensors, ctx.eps, *ctx.needs_input_grad[:3]), None)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """weight * (x - mean) / sqrt(variance + eps) + bias over the last axis of x, rounded once to its type; differentiable, once, in x, weight
    and bias.  x float32, float16 or bfloat16, of at most 16384 elements along that axis; weight and bias (d,), float32 or of x's type."""
    if forward_ad._current_level >= 0 or (torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or
                                                                       (bias is not None and bias.requires_grad))):
        return _LayerNorm.apply(x, weight, bias, float(eps))
    return _norm_forward(x, weight, bias, float(eps))


# ------------------------------------------------------------------------------------------------ sampling
def _setting(name, value, rows, dtype, device):
    """(pointer, value for all rows): a tensor holds one for each row."""
    if isinstance(value, torch.Tensor):
        if value.shape != (rows,) or value.dtype != dtype or not value.is_contiguous() or value.device != device:
            raise ValueError(f"{name}: a number, or a contiguous {dtype} tensor of one value for each row, on the device of the logits")
        return value.data_ptr(), 0
    if value != value:
        raise ValueError(f"{name} is {value}")
    return 0, value


def sample(logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, output_log_prob=False):
    """One token for each row of logits (rows, vocabulary), float32, float16 or bfloat16: int64 (rows,); with ``output_log_prob=True`` also the log
    of the probability that it was drawn with, float32.

    Every token has the weight exp((logit - largest) / temperature).  In the order of falling logits, the lower token first among
    equals, the first `top_k` are kept (0: all), as far as their weight is at least `min_p`, and of these the fewest whose weights add up
    to `top_p` of the weight of them all; at least one.  `uniform` (rows,), float32 or float64 from [0, 1), picks the token: the first, in the order of tokens,
    with which the kept weights add up to more than that part of their sum.  temperature 0 takes the largest logit, the lowest token
    among equals.  The settings are numbers, or a tensor with one for each row (float32; top_k: int32).  NaN counts as minus infinity; a row that holds
    nothing above it gives -1.  No gradient is computed: with gradients enabled, logits that require one are refused."""
    if forward_ad._current_level >= 0:
        _no_tangents(logits=logits, uniform=uniform)
    if torch.is_grad_enabled():
        _not_recorded(logits=logits)
    dtype, device = logits.dtype, logits.device
    if dtype not in _FLOAT:
        raise TypeError(f"sampling takes float32, float16 or bfloat16, not {dtype}")
    if logits.dim() != 2 or logits.shape[1] == 0:
        raise ValueError(f"logits: (rows, vocabulary), not {tuple(logits.shape)}")
    rows, vocabulary = logits.shape
    if uniform.shape != (rows,) or uniform.dtype not in (torch.float32, torch.float64) or not uniform.is_contiguous() or uniform.device != device:
        raise ValueError("uniform: a contiguous float32 or float64 tensor of one value for each row, on the device of the logits")
    d_temperature, temperature = _setting("temperature", temperature, rows, torch.float32, device)
    d_top_k, top_k = _setting("top_k", top_k, rows, torch.int32, device)
    d_top_p, top_p = _setting("top_p", top_p, rows, torch.float32, device)
    d_min_p, min_p = _setting("min_p", min_p, rows, torch.float32, device)
    if not 0.0 <= temperature < float("inf"):
        raise ValueError(f"temperature is {temperature}")
    if vocabulary > 1 and logits.stride(1) != 1:
        logits = logits.contiguous()
    tokens = logits.new_empty(rows, dtype=torch.int64)
    log_prob = None
    if output_log_prob:
        log_prob = torch.empty_like(uniform) if uniform.dtype == torch.float32 else logits.new_empty(rows, dtype=torch.float32)
    args = B.tcu_sample_args(_FLOAT[dtype], rows, vocabulary, logits.data_ptr(), logits.stride(0), uniform.data_ptr(), int(uniform.dtype == torch.float64), tokens.data_ptr(),
                             _ptr(log_prob), d_temperature=d_temperature, d_top_k=d_top_k, d_top_p=d_top_p, d_min_p=d_min_p, temperature=float(temperature),
                             top_k=min(max(int(top_k), 0), 1 << 40), top_p=float(top_p), min_p=float(min_p))
    B.check(B.tcu_sample(args, _stream(device)))
    return (tokens, log_prob) if output_log_prob else tokens
