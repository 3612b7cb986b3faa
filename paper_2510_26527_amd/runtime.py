"""Device-memory plumbing around the C boundary: owns the torch tensors a handle points at.

Nothing here computes; each method allocates or copies tensors and forwards to the binding
function of the same name in the package root.
"""
import torch

import paper_2510_26527_amd as psd

_LAYER_WEIGHTS = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")
_QUANT_WEIGHTS = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


def weight_order(n_layers):
    names = ["embed"]
    for l in range(n_layers):
        names += [f"l{l}.{n}" for n in _LAYER_WEIGHTS]
    return names + ["final_norm", "lm_head"]


class Model:
    """A psd_model handle plus the weight tensors it points at (kept alive here)."""

    def __init__(self, shape, weights, device="cuda", quant=None):
        # shape: any object with the psd_model_desc field names; weights: name -> tensor
        # quant: for a 4-bit model, name -> (scale bf16 [n, K/128], zero uint8 [n, K/128]) for every projection;
        #        weights[name] then holds the codes, uint8 [n, K/2]
        dt = weights["embed"].dtype
        self.dtype = dt
        self.code = psd.dtype_code(dt)
        self.device = torch.device(device)
        self.weights = {k: v.to(self.device).contiguous() for k, v in weights.items()}
        self.desc = psd.psd_model_desc(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads,
                                       shape.d_head, shape.d_ffn, shape.vocab, shape.rope_theta, shape.rms_eps,
                                       self.code)
        self.shape = shape
        ptrs = [self.weights[n].data_ptr() for n in weight_order(shape.n_layers)]
        self.quant = None
        if quant is None:
            self.handle = psd.psd_model_create(self.desc, ptrs)
        else:
            self.quant = {k: (s.to(self.device).contiguous(), z.to(self.device).contiguous()) for k, (s, z) in quant.items()}
            names = [f"l{l}.{n}" for l in range(shape.n_layers) for n in _QUANT_WEIGHTS]
            self.handle = psd.psd_model_create_w4(self.desc, ptrs, [self.quant[n][0].data_ptr() for n in names],
                                                  [self.quant[n][1].data_ptr() for n in names])
        self._ws = None
        self.packed = None
        self.rope = None

    def set_rope(self, rope):
        """Turn by `rope` (a Rope, None: by the shape's rope_theta) in every forward from now on."""
        psd.psd_model_set_rope(self.handle, None if rope is None else rope.handle)
        self.rope = rope
        return self

    def pack(self):
        """Build the streaming copy of the projection weights (bf16 models) for steps of up to 128 rows."""
        need = psd.psd_model_packed_bytes(self.handle)
        if need == 0:
            return self
        self.packed = torch.empty(need, dtype=torch.uint8, device=self.device)
        psd.psd_model_pack(self.handle, self.packed)
        self._ws = None
        return self

    def workspace(self, batch, n_new, max_len):
        need = psd.psd_model_workspace_bytes(self.handle, batch, n_new, max_len)
        if need == 0:
            raise ValueError("unsupported batch / n_new / max_len")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def workspace_upto(self, batch, max_new, max_len):
        """A workspace large enough for every n_new in 1..max_new."""
        need = max(psd.psd_model_workspace_bytes(self.handle, batch, r, max_len) for r in range(1, max_new + 1))
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def close(self):
        if self.handle is not None:
            psd.psd_model_destroy(self.handle)
            self.handle = None


class KVCache:
    """K [L,B,h_kv,max_len,d_h] and transposed V [L,B,h_kv,d_h,max_len] tensors, the device
    length vector, and the psd_kv handle over them."""

    def __init__(self, model: Model, batch, max_len, fill_garbage=False):
        s = model.shape
        self.model, self.batch, self.max_len = model, batch, max_len
        alloc = torch.empty if not fill_garbage else (lambda *a, **k: torch.full(*a, float("nan"), **k))
        self.k = alloc((s.n_layers, batch, s.n_kv_heads, max_len, s.d_head), dtype=model.dtype, device=model.device)
        self.v = alloc((s.n_layers, batch, s.n_kv_heads, s.d_head, max_len), dtype=model.dtype, device=model.device)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=model.device)
        self.handle = psd.psd_kv_create(model.handle, batch, max_len, self.k, self.v, self.lens, 0)

    def load(self, k_layers, v_layers, lens):
        """Copy given contents in: k_layers / v_layers are per-layer [B, h_kv, n_ctx, d_h] tensors
        (logical layout), lens the valid length per sequence (int or list)."""
        n_ctx = k_layers[0].shape[2]
        for l, (k, v) in enumerate(zip(k_layers, v_layers)):
            self.k[l, :, :, :n_ctx].copy_(k)
            self.v[l, :, :, :, :n_ctx].copy_(v.transpose(-1, -2))
        lens_t = torch.as_tensor(lens, dtype=torch.int32).expand(self.batch).contiguous()
        self.lens.copy_(lens_t)
        psd.psd_kv_destroy(self.handle)
        self.handle = psd.psd_kv_create(self.model.handle, self.batch, self.max_len, self.k, self.v, self.lens,
                                        int(lens_t.max()))

    def close(self):
        if self.handle is not None:
            psd.psd_kv_destroy(self.handle)
            self.handle = None


_CODE = {torch.float32: psd.PSD_F32, torch.bfloat16: psd.PSD_BF16}


def _current(*tensors):
    """The library enqueues on the current device: a tensor of another one is the caller's mistake.  -> the current device."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t.get_device() != here:
            raise ValueError(f"tensor on {t.device}, the current device is cuda:{here}")
    return here


_raw = torch._C._cuda_getCurrentRawStream                    # a device's current stream, without a Stream object


def _code(dtype):
    code = _CODE.get(dtype)
    if code is None:
        raise ValueError(f"float32 or bfloat16 expected, not {dtype}")
    return code


def _made_on(stream, make, *args, **kw):
    """A new tensor for `stream` (None: the current one) to write: what its memory held before must be done with on that stream."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        return make(*args, **kw)


def _row_stride(t):
    """Elements between the rows of t [..., heads, d], whose heads are dense within a row, and rows evenly apart."""
    shape = t.shape
    width = shape[-2] * shape[-1]
    if t.is_contiguous():
        return width
    strides = t.stride()
    if strides[-1] != 1 or (shape[-2] > 1 and strides[-2] != shape[-1]):
        raise ValueError("a row's heads have to lie side by side")
    stride, span = None, 1
    for k in range(len(shape) - 3, -1, -1):
        if shape[k] > 1:
            if stride is None:
                stride = strides[k]
            elif strides[k] != stride * span:
                raise ValueError("rows have to be evenly apart")
            span *= shape[k]
    return width if stride is None else stride


def _row_stride4(t, n, d):
    """_row_stride of t [B, n, heads, d], first for one piece or the heads of a buffer of projections."""
    s0, s1, s2, s3 = t.stride()
    return s1 if s3 == 1 and s2 == d and s0 == s1 * n else _row_stride(t)


class Rope:
    """A psd_rope: how query and key heads turn by their positions."""

    _LAYOUT = {"half": psd.PSD_ROPE_HALF, "interleaved": psd.PSD_ROPE_INTERLEAVED}
    _SCALING = {"none": psd.PSD_ROPE_PLAIN, "linear": psd.PSD_ROPE_LINEAR, "base": psd.PSD_ROPE_BASE, "parts": psd.PSD_ROPE_PARTS}

    def __init__(self, d_head, rot_dim=None, layout="half", theta=1.0e4, scaling="none", factor=1.0, low=1.0, high=4.0,
                 original_len=0, magnitude=1.0):
        self._handle = None
        self.d_head, self.rot_dim = d_head, d_head if rot_dim is None else rot_dim
        self._handle = psd.psd_rope_create(psd.psd_rope_desc(d_head, self.rot_dim, self._LAYOUT[layout], self._SCALING[scaling], theta,
                                                            factor, low, high, original_len, magnitude))

    @property
    def handle(self):
        if self._handle is None:                             # (no handle would mean: nothing turns)
            raise ValueError("this Rope was closed")
        return self._handle

    def frequencies(self):
        return psd.psd_rope_frequencies(self.handle, self.rot_dim // 2)

    def rotate(self, x, positions, out=None, stream=None):
        """x [..., heads, d_head] (fp32 or bf16), positions int32 of its leading shape -> a new tensor, or `out` (which may be x)."""
        shape = x.shape
        if shape[:-2] != positions.shape or shape[-1] != self.d_head or positions.dtype != torch.int32 or not positions.is_contiguous():
            raise ValueError("x [..., heads, d_head] with contiguous int32 positions [...] expected")
        if out is None:
            out = _made_on(stream, torch.empty_like, x)
        elif out.shape != shape or out.dtype != x.dtype:
            raise ValueError("out has another shape or type than x")
        here = _current(x, positions, out)
        rows = positions.numel()
        if rows:
            psd.psd_rope_rotate(self.handle, x, out, positions, rows, shape[-2], _code(x.dtype), _row_stride(x), _row_stride(out),
                                _raw(here) if stream is None else stream)
        return out

    def close(self):
        if self._handle is not None:
            psd.psd_rope_destroy(self._handle)
            self._handle = None


class KVCache8:
    """An 8-bit cache: e4m3 codes k [L,B,h_kv,max_len,d_h] and v [L,B,h_kv,max_len/64,d_h,64], their scales [L,B,h_kv,max_len/64],
    the device length vector, and the psd_kv handle over them.  Goes wherever a KVCache goes, but for token trees."""

    def __init__(self, model: Model, batch, max_len, fill_garbage=False):
        s = model.shape
        self.model, self.batch, self.max_len = model, batch, max_len
        lead = (s.n_layers, batch, s.n_kv_heads)
        make = (lambda shape, dt: torch.full(shape, 255 if dt == torch.uint8 else float("nan"), dtype=dt, device=model.device)) \
            if fill_garbage else (lambda shape, dt: torch.empty(shape, dtype=dt, device=model.device))
        self.k = make(lead + (max_len, s.d_head), torch.uint8)
        self.v = make(lead + (max_len // 64, s.d_head, 64), torch.uint8)
        self.k_scale = make(lead + (max_len // 64,), torch.float32)
        self.v_scale = make(lead + (max_len // 64,), torch.float32)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=model.device)
        self._create(0)

    def _create(self, bound):
        self.handle = psd.psd_kv_create_q8(self.model.handle, self.batch, self.max_len, self.k, self.v, self.k_scale, self.v_scale,
                                           self.lens, bound)

    def load(self, k_layers, v_layers, lens):
        """Quantise given contents in: per-layer [B, h_kv, n_ctx, d_h] tensors whose keys are rotated already, lens the valid length
        per sequence (int or list)."""
        n_ctx = k_layers[0].shape[2]
        self.lens.zero_()
        psd.psd_kv_destroy(self.handle)
        self.handle = None
        self._create(0)
        for l, (k, v) in enumerate(zip(k_layers, v_layers)):
            rows = [t.to(self.model.device).transpose(1, 2).contiguous() for t in (k, v)]
            if n_ctx:
                self.layer(l).append(None, rows[0], rows[1], None, len_upper_bound=n_ctx)
        lens_t = torch.as_tensor(lens, dtype=torch.int32).expand(self.batch).contiguous()
        self.lens.copy_(lens_t)
        psd.psd_kv_destroy(self.handle)
        self.handle = None
        self._create(int(lens_t.max()))

    def layer(self, l):
        """One layer, for programs that append and attend by themselves."""
        return KV8Layer(self.k[l], self.v[l], self.k_scale[l], self.v_scale[l], self.lens)

    def close(self):
        if self.handle is not None:
            psd.psd_kv_destroy(self.handle)
            self.handle = None


class KV8Layer:
    """One layer of an 8-bit cache over the caller's tensors: codes uint8 k [B, h_kv, max_len, d_h] and v [B, h_kv, max_len/64, d_h, 64],
    scales fp32 [B, h_kv, max_len/64], lens int32 [B]."""

    def __init__(self, k, v, k_scale, v_scale, lens):
        B, h, n, d = k.shape
        if tuple(v.shape) != (B, h, n // 64, d, 64) or tuple(k_scale.shape) != (B, h, n // 64) or k_scale.shape != v_scale.shape:
            raise ValueError("codes and scales do not belong together")
        if k.dtype != torch.uint8 or v.dtype != torch.uint8 or k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32:
            raise ValueError("codes are uint8, scales float32")
        if tuple(lens.shape) != (B,) or lens.dtype != torch.int32 or not all(t.is_contiguous() and t.device == k.device for t in (k, v, k_scale, v_scale, lens)):
            raise ValueError("lens is int32 [B], and every tensor contiguous and on one device")
        self.k, self.v, self.k_scale, self.v_scale, self.lens = k, v, k_scale, v_scale, lens
        self.dims = B, h, d
        self.view = psd.psd_kv8_view(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), lens.data_ptr(), B, h, d, n)

    def append(self, q, k, v, rope=None, len_upper_bound=None, q_out=None, stream=None):
        """Rows q [B, n_new, h_q, d_h] (or None), k and v [B, n_new, h_kv, d_h], all fp32 or all bf16, at positions lens[b] ..: rotated
        by `rope` and quantised into the cache -> the rotated queries.  len_upper_bound: a bound of lens[b] + n_new."""
        shape, dtype = k.shape, k.dtype
        B, n, h, d = shape
        if (B, h, d) != self.dims or v.shape != shape or v.dtype != dtype:
            raise ValueError("k and v are [B, n_new, n_kv_heads, d_head] of one type")
        q_stride, out_stride, h_q = 0, 0, h
        if q is None:
            q_out = None
            here = _current(k, v, self.k)
        else:
            q_shape = q.shape
            h_q = q_shape[2]
            if q_shape != (B, n, h_q, d) or q.dtype != dtype:
                raise ValueError("q is [B, n_new, n_q_heads, d_head] of k's type")
            if q_out is None:
                q_out = _made_on(stream, torch.empty_like, q)
            elif q_out.shape != q_shape or q_out.dtype != dtype:
                raise ValueError("q_out has another shape or type than q")
            here = _current(k, v, self.k, q, q_out)
            q_stride, out_stride = _row_stride4(q, n, d), _row_stride4(q_out, n, d)
        psd.psd_kv8_append(self.view, None if rope is None else rope.handle, q, k, v, q_out, n, h_q, _code(dtype), q_stride,
                           _row_stride4(k, n, d), _row_stride4(v, n, d), out_stride,
                           self.view.max_len if len_upper_bound is None else len_upper_bound, _raw(here) if stream is None else stream)
        return q_out


class KV8Attention:
    """Workspace of psd_kv8_attention, reused across calls (on one stream at a time).  One that was outgrown is kept, since a captured
    graph may point at it; each is at least twice its predecessor (of the same device)."""

    def __init__(self):
        self._ws = None
        self._outgrown = []

    def __call__(self, cache: KV8Layer, q, scale=0.0, len_upper_bound=None, out=None, stream=None):
        """q bf16 [B, n_new, h_q, d_h], the rows just appended to `cache` -> bf16 of the same shape; scale 0: 1 / sqrt(d_h).
        len_upper_bound: a bound of lens[b] + n_new."""
        view, shape = cache.view, q.shape
        B, n, h_q, d = shape
        if B != cache.dims[0] or d != cache.dims[2] or q.dtype != torch.bfloat16:
            raise ValueError("q is bf16 [B, n_new, n_q_heads, d_head]")
        if out is None:
            out = _made_on(stream, torch.empty_like, q)
        elif out.shape != shape or out.dtype != torch.bfloat16:
            raise ValueError("out has another shape or type than q")
        here = _current(q, cache.k, out)
        bound = view.max_len if len_upper_bound is None else len_upper_bound
        q_stride, out_stride = _row_stride4(q, n, d), _row_stride4(out, n, d)
        if self._ws is not None and self._ws.get_device() != here:
            self._outgrown.append(self._ws)
            self._ws = None
        queue = _raw(here) if stream is None else stream
        for grown in (False, True):
            try:
                psd.psd_kv8_attention(view, q, out, n, h_q, scale, q_stride, out_stride, bound, self._ws, queue)
                return out
            except psd.PsdError as e:                        # too small a workspace so far: nothing was enqueued
                if grown or e.status != psd.PSD_ERR_WORKSPACE:
                    raise
                need = psd.psd_kv8_attention_workspace_bytes(B, n, h_q, view.n_kv_heads, d, bound)
                if self._ws is not None:
                    self._outgrown.append(self._ws)
                    need = max(need, 2 * self._ws.numel())
                self._ws = _made_on(stream, torch.empty, need, dtype=torch.uint8, device=q.device)


def forward(model: Model, kv: KVCache, tokens, n_logit_rows=None, logits_out=None, stream=None):
    """tokens int32 [B, n_new] on the device -> fp32 logits [B, n_logit_rows, V] (a new tensor
    unless logits_out is given)."""
    B, n_new = tokens.shape
    rows = n_new if n_logit_rows is None else n_logit_rows
    if logits_out is None and rows > 0:
        logits_out = torch.empty((B, rows, model.shape.vocab), dtype=torch.float32, device=model.device)
    ws = model.workspace(B, n_new, kv.max_len)
    psd.psd_model_forward(model.handle, tokens, n_new, kv.handle, logits_out, rows, ws, stream)
    return logits_out


def forward_tree(model: Model, kv: KVCache, tokens, parents, logits_out=None, stream=None):
    """tokens int32 [B, n_nodes] on the device, parents a host sequence (parents[0] = -1, parents[i] < i) ->
    fp32 logits [B, n_nodes, V]."""
    B, n = tokens.shape
    if logits_out is None:
        logits_out = torch.empty((B, n, model.shape.vocab), dtype=torch.float32, device=model.device)
    ws = model.workspace(B, n, kv.max_len)
    psd.psd_model_forward_tree(model.handle, tokens, n, parents, kv.handle, logits_out, ws, stream)
    return logits_out


def tree_accept(p_logits, q_logits, tokens, parents, uniforms, temperature=1.0, stream=None):
    """p, q [rows, n_nodes, V] (same dtype; q may be None when temperature is 0), tokens int32 [rows, n_nodes],
    uniforms fp32 [rows, n_nodes + 1] -> (path_len [rows], path [rows, n_nodes], token [rows], flags [rows]) int32."""
    rows, n, V = p_logits.shape
    dev = p_logits.device
    out_len = torch.empty(rows, dtype=torch.int32, device=dev)
    out_path = torch.full((rows, n), -1, dtype=torch.int32, device=dev)
    out_tok = torch.empty(rows, dtype=torch.int32, device=dev)
    out_flags = torch.empty(rows, dtype=torch.int32, device=dev)
    psd.psd_tree_accept(p_logits, q_logits, tokens, parents, n, uniforms, temperature, out_len, out_path, out_tok, rows, V,
                        psd.dtype_code(p_logits.dtype), p_logits.stride(0), q_logits.stride(0) if q_logits is not None else 0,
                        out_flags, stream)
    return out_len, out_path, out_tok, out_flags


class Acceptor:
    """Output tensors and workspace of psd_spec_accept, reused across calls."""

    def __init__(self, device="cuda"):
        self.device = torch.device(device)
        self._ws = None
        self._out = None

    def __call__(self, p_logits, q_logits, draft_tokens, uniforms, temperature=1.0, stream=None):
        """p [rows, n_p_rows, V], q [rows, gamma, V] (same dtype), tokens int32 [rows, gamma],
        uniforms fp32 [rows, gamma+1] -> (accept_len, token, flags) int32 [rows] tensors."""
        rows, n_p_rows, V = p_logits.shape
        gamma = uniforms.shape[1] - 1
        need = psd.psd_spec_accept_workspace_bytes(rows, gamma, n_p_rows, V)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        if self._out is None or self._out.shape[1] < rows:
            self._out = torch.empty((3, max(rows, 1)), dtype=torch.int32, device=self.device)
        n, tok, fl = self._out[0, :rows], self._out[1, :rows], self._out[2, :rows]
        q_stride = q_logits.stride(0) if gamma > 0 and q_logits is not None else 0
        psd.psd_spec_accept(p_logits, q_logits if gamma > 0 else None, draft_tokens if gamma > 0 else None, gamma,
                            uniforms, temperature, n, tok, rows, n_p_rows, V, psd.dtype_code(p_logits.dtype),
                            p_logits.stride(0), q_stride, fl, self._ws, stream)
        return n, tok, fl
