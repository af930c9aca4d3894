"""Autograd modules over the lmbp kernels, and the affine merge that enables MS-BP.

* ``ReGELU2`` / ``ReSiLU2``: exact GELU / SiLU forward, 2-bit codes saved, step
  derivative backward (Sec. 4.2).
* ``ReSwiGLU2``: h = SiLU(g) * u with ReSiLU2's backward for the SiLU factor (the LLaMA
  MLP, Sec. 6); saves the codes and s = SiLU(g).
* ``MSLayerNorm`` / ``MSRMSNorm``: parameter-free norms (Sec. 5.2, Appendix G) that save
  only their output z and one fp32 rstd per row. z is the same tensor the following
  linear layer saves as its input, so autograd keeps one copy (memory sharing).
* ``LinearReGELU2`` / ``LinearReSiLU2``: a bf16 linear layer followed by the activation,
  forward fused into one kernel (the pre-activation is never stored); saves x (for the
  weight gradient) and the codes. Backward: dz = dy * slope[code] with the bias gradient
  in one kernel, the weight gradient in another, the input's product by a library GEMM.
* ``LinearReSwiGLU2``: the LLaMA MLP's gate and up projections with SwiGLU, forward fused
  in one kernel (g never stored); backward through the SwiGLU activation backward and
  the linear layers' products.
* ``LinearQ8``: a linear layer whose frozen weight is kept in 8 bits (one scale per output
  channel); its input's rows are brought to 8 bits and the product runs on whole numbers.
  Keeps nothing of its input.
* ``MSRMSNormLinearQ8``: residual addition, MS-RMSNorm with its output in 8 bits, and the
  ``LinearQ8`` layers that consume it. Keeps one byte per element of the norm's output and
  two fp32 values per row for the norm's backward; the frozen layers keep nothing of it. The
  output z itself is not handed out: where something else reads it (an adapter beside a
  layer), ``MSRMSNorm`` and ``LinearQ8`` are the pair to use, and z stays in its own type.
* ``Rope``: rotary positions of query and key heads (one or several axes); keeps nothing but the positions.
* ``MSRMSNormRope``: RMSNorm of each query and key head and the rotation in one pass. Without gains it keeps its
  outputs, which attention keeps anyway, and one fp32 rstd per head: the rotation keeps products, so the norm's
  backward works from them as it is. With gains it keeps its inputs instead.
* ``Attention``: softmax(scale q k^T) v of bf16 heads, causal or not, grouped heads, equal or packed sequences;
  keeps q, k, v, its output and one fp32 value per row.
* ``QKVAttention``: rotation (with the norm of the heads in front, if asked for) and attention on the one output of a
  fused projection, as one node: the gradients are written into one tensor.
* ``merge_norm_into_linears``: folds a norm's affine (alpha, beta) into the linear layers
  that consume its output, W~ = W diag(alpha), b~ = W beta + b (Sec. 5.2), and returns
  the parameter-free MS norm to use in its place.

The modules answer in the type of their input (fp32 or bf16, the fused linear layers bf16 alone) and
refuse others, inside an autocast region as outside: autocast casts nothing for them.

Every forward and backward runs in the HIP kernels through ``binding``, except the
product of the fused linear layers' backward for the input (torch's library GEMM) and
the one-time weight merge.
"""

import torch
from torch import nn

from . import binding


def _flat(t):
    return t if t.is_contiguous() else t.contiguous()


class _Act(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, which):
        fwd = binding.regelu2_fwd if which == "gelu" else binding.resilu2_fwd
        y, codes = fwd(_flat(x))
        ctx.which = which
        ctx.save_for_backward(codes)
        return y

    @staticmethod
    def backward(ctx, dy):
        (codes,) = ctx.saved_tensors
        bwd = binding.regelu2_bwd if ctx.which == "gelu" else binding.resilu2_bwd
        return bwd(_flat(dy), codes), None


class _SwiGLU(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, u):
        g, u = _flat(g), _flat(u)
        if g.shape != u.shape:
            raise ValueError("g and u must have the same shape")
        h, s, codes = binding.reswiglu2_fwd(g, u)
        ctx.save_for_backward(u, s, codes)
        return h

    @staticmethod
    def backward(ctx, dh):
        u, s, codes = ctx.saved_tensors
        dg, du = binding.reswiglu2_bwd(_flat(dh), u, s, codes)
        return dg, du


class _MSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, eps, centered):
        fwd = binding.msln_fwd if centered else binding.msrms_fwd
        z, rstd = fwd(_flat(x), eps)
        ctx.centered = centered
        ctx.save_for_backward(z, rstd)
        return z

    @staticmethod
    def backward(ctx, dz):
        z, rstd = ctx.saved_tensors
        bwd = binding.msln_bwd if ctx.centered else binding.msrms_bwd
        return bwd(_flat(dz), z, rstd), None, None


def _in_kernels(dz, x2):
    """Whether the parameters' gradients can come from the library's kernels: not when the
    backward pass is itself being recorded (create_graph: torch's products then carry the
    graph), nor for tensors that a saved-tensor hook gave back in another layout."""
    return (not torch.is_grad_enabled() and dz.is_contiguous() and x2.is_contiguous()
            and dz.dtype == x2.dtype == torch.bfloat16 and dz.device == x2.device
            and dz.data_ptr() % 16 == 0 and x2.data_ptr() % 16 == 0
            and 0 < dz.shape[1] <= 1 << 24 and 0 < x2.shape[1])


def _weight_grad(dz, x2):
    return binding.linear_weight_grad(dz, x2) if _in_kernels(dz, x2) else dz.t().mm(x2)


def _two_products(a, b, c, d):
    """a b + c d. The second product is added in place (out of place the first one is copied
    before), except under autocast, which casts no operand of an in-place call."""
    first = a @ b
    if torch.is_autocast_enabled(first.device.type):
        return torch.addmm(first, c, d)
    return first.addmm_(c, d)


class _LinearAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, which):
        x2 = _flat(x).reshape(-1, x.shape[-1])
        y, codes = binding.linear_act_fwd(x2, _flat(weight), None if bias is None else _flat(bias),
                                          act=which)
        ctx.which = which
        ctx.has_bias = bias is not None
        ctx.x_shape = x.shape
        ctx.save_for_backward(x2, weight, codes)
        return y.reshape(*x.shape[:-1], weight.shape[0])

    @staticmethod
    def backward(ctx, dy):
        x2, weight, codes = ctx.saved_tensors
        dy = _flat(dy).reshape(-1, weight.shape[0])
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        need_b = ctx.has_bias and need_b
        if need_b and _in_kernels(dy, x2):
            dz, dw, db = binding.linear_act_bwd(dy, codes, x2, ctx.which, weight_grad=need_w)
        else:
            dz = (binding.regelu2_bwd if ctx.which == "gelu" else binding.resilu2_bwd)(dy, codes)
            dw = _weight_grad(dz, x2) if need_w else None
            db = dz.sum(0, dtype=torch.float32).to(dz.dtype) if need_b else None
        # The input's product as torch's own linear layer forms it (a 2-D library GEMM).
        dx = (dz @ weight).reshape(ctx.x_shape) if need_x else None
        return dx, dw, db, None


class _LinearActModule(nn.Linear):
    """bf16 nn.Linear whose output goes through the activation, fused. Output features
    must be a multiple of 16, input features a multiple of 8."""
    which = None

    def __init__(self, in_features, out_features, bias=True, device=None, dtype=torch.bfloat16):
        super().__init__(in_features, out_features, bias=bias, device=device, dtype=dtype)

    def forward(self, x):
        return _LinearAct.apply(x, self.weight, self.bias, self.which)


class LinearReGELU2(_LinearActModule):
    """GELU(x W^T + b) with ReGELU2's backward (Sec. 4.2), forward fused in one kernel."""
    which = "gelu"


class LinearReSiLU2(_LinearActModule):
    """SiLU(x W^T + b) with ReSiLU2's backward (Sec. 4.2), forward fused in one kernel."""
    which = "silu"


class _LinearSwiGLU(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up):
        x2 = _flat(x).reshape(-1, x.shape[-1])
        h, s, u, codes = binding.linear_swiglu_fwd(x2, _flat(w_gate), _flat(w_up))
        ctx.x_shape = x.shape
        ctx.save_for_backward(x2, w_gate, w_up, s, u, codes)
        return h.reshape(*x.shape[:-1], w_gate.shape[0])

    @staticmethod
    def backward(ctx, dh):
        x2, w_gate, w_up, s, u, codes = ctx.saved_tensors
        dg, du = binding.reswiglu2_bwd(_flat(dh).reshape(-1, w_gate.shape[0]), u, s, codes)
        dx = _two_products(dg, w_gate, du, w_up).reshape(ctx.x_shape) if ctx.needs_input_grad[0] else None
        dwg = _weight_grad(dg, x2) if ctx.needs_input_grad[1] else None
        dwu = _weight_grad(du, x2) if ctx.needs_input_grad[2] else None
        return dx, dwg, dwu


class LinearReSwiGLU2(nn.Module):
    """The LLaMA MLP's input side, SiLU(x Wg^T) * (x Wu^T), with ReSiLU2's backward for
    the SiLU factor; forward fused in one kernel (bf16; out_features a multiple of 16,
    in_features of 8). Saves x, s = SiLU(g), u and the codes of g."""

    def __init__(self, in_features, out_features, device=None, dtype=torch.bfloat16):
        super().__init__()
        self.gate = nn.Linear(in_features, out_features, bias=False, device=device, dtype=dtype)
        self.up = nn.Linear(in_features, out_features, bias=False, device=device, dtype=dtype)

    def forward(self, x):
        return _LinearSwiGLU.apply(x, self.gate.weight, self.up.weight)


class ReGELU2(nn.Module):
    """GELU forward; backward through the 2-bit step derivative (Sec. 4.2)."""

    def forward(self, x):
        return _Act.apply(x, "gelu")


class ReSiLU2(nn.Module):
    """SiLU forward; backward through the 2-bit step derivative (Sec. 4.2)."""

    def forward(self, x):
        return _Act.apply(x, "silu")


class ReSwiGLU2(nn.Module):
    """h = SiLU(g) * u with ReSiLU2's backward for the SiLU factor."""

    def forward(self, g, u):
        return _SwiGLU.apply(g, u)


class MSLayerNorm(nn.Module):
    """LayerNorm without affine over the last dimension, saving only z and rstd
    (Alg. 1 / Alg. 2). Use after merging the affine into the next linear layers."""

    def __init__(self, eps=1e-6):
        super().__init__()
        self.eps = float(eps)

    def forward(self, x):
        return _MSNorm.apply(x, self.eps, True)

    def extra_repr(self):
        return f"eps={self.eps}"


class MSRMSNorm(nn.Module):
    """RMSNorm without weight over the last dimension, saving only z and rstd (Alg. 3)."""

    def __init__(self, eps=1e-5):
        super().__init__()
        self.eps = float(eps)

    def forward(self, x):
        return _MSNorm.apply(x, self.eps, False)

    def extra_repr(self):
        return f"eps={self.eps}"


class _LinearQ8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, scale, bias):
        x2 = _flat(x).reshape(-1, x.shape[-1])
        q, q_scale = binding.q8_rows(x2)
        ctx.bias_dtype = bias.dtype if bias is not None else None
        ctx.save_for_backward(weight, scale)
        return _product_q8(q, q_scale, weight, scale, bias, x.dtype).reshape(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        weight, scale = ctx.saved_tensors
        dx = _input_grad_q8(dy, weight, scale, dy.dtype) if ctx.needs_input_grad[0] else None
        return dx, None, None, _bias_grad(dy, ctx.bias_dtype) if ctx.needs_input_grad[3] else None


def _product_q8(q, q_scale, weight, scale, bias, dtype):
    if bias is not None:
        bias = _flat(bias if bias.dtype == dtype else bias.to(dtype))
    return binding.linear_q8_fwd(q, q_scale, weight, scale, bias, dtype)


def _input_grad_q8(dy, weight, scale, dtype, add=None):
    """dx = (dy scale) weight + add in ``dtype`` (in add's place, if there is one). Of more output channels
    than one sum holds, in shares of whole 64s (w's rows stay aligned): each brings its part of dy's rows to 8 bits,
    with a scale of its own, and they add up in fp32."""
    n = weight.shape[0]
    if n <= binding.Q8_MAX_SUM:
        return binding.linear_q8_bwd(_flat(dy), weight, scale, add=add, dx=add, dtype=dtype)
    shares = -(-n // (binding.Q8_MAX_SUM // 64 * 64))
    size = -(-n // (64 * shares)) * 64
    dx = add
    for at in range(0, n, size):
        part = slice(at, at + size)
        dx = binding.linear_q8_bwd(_flat(dy[..., part]), weight[part], scale[part], add=dx, dx=dx, dtype=torch.float32)
    return dx.to(dtype)


def _bias_grad(dy, dtype):
    kept = dtype if dtype in (torch.float32, torch.bfloat16) else torch.float32
    return binding.linear_bias_grad(_flat(dy), kept).to(dtype)


class LinearQ8(nn.Module):
    """Linear layer with a frozen 8-bit weight: ``weight`` int8 [n, k] and ``scale`` fp32 [n]
    (buffers; w = weight * scale), ``bias`` [n] or None (a parameter, frozen unless its
    ``requires_grad`` is set). The input's rows are brought to 8 bits, and so are the rows of
    the output's gradient in the backward; nothing of the input is kept. k is at most 131071 (a sum
    in 32 bits), n any number: the gradient of more than 131071 outputs is that of several layers."""

    def __init__(self, weight, scale, bias=None):
        super().__init__()
        if weight.dtype != torch.int8 or weight.dim() != 2:
            raise ValueError("weight must be an int8 tensor [n, k]")
        if scale.dtype != torch.float32 or scale.shape != weight.shape[:1]:
            raise ValueError("scale must be a float32 tensor [n]")
        if bias is not None and bias.shape != weight.shape[:1]:
            raise ValueError("bias must have n elements")
        self.register_buffer("weight", weight.contiguous())
        self.register_buffer("scale", scale.contiguous())
        self.bias = None if bias is None else nn.Parameter(bias.detach().clone(), requires_grad=False)

    @classmethod
    @torch.no_grad()
    def from_linear(cls, linear):
        """The 8-bit form of a linear layer on the GPU (after merging a norm's affine, if any)."""
        weight, scale = binding.q8_rows(_flat(linear.weight.detach()))
        return cls(weight, scale, linear.bias)

    @property
    def in_features(self):
        return self.weight.shape[1]

    @property
    def out_features(self):
        return self.weight.shape[0]

    def _apply(self, fn, recurse=True):
        scale = self.scale
        super()._apply(fn, recurse)
        if self.scale.dtype != torch.float32:   # a change of the model's type is not meant for the scales
            self.scale = scale.to(self.scale.device)
        return self

    def values(self, dtype=torch.bfloat16):
        """The weight that the layer computes with, in ``dtype``."""
        return binding.q8_values(self.weight, self.scale, dtype)

    def forward(self, x):
        return _LinearQ8.apply(x, self.weight, self.scale, self.bias)

    def extra_repr(self):
        return f"in_features={self.in_features}, out_features={self.out_features}, bias={self.bias is not None}"


class _NormLinearQ8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, res, eps, *layers):
        out = binding.msrms_q8_fwd(_flat(x), eps, None if res is None else _flat(res))
        q, q_scale, rstd = out[:3]
        ctx.set_materialize_grads(False)
        ctx.dtype = x.dtype
        ctx.bias_dtypes = [b.dtype if b is not None else None for b in layers[2::3]]
        ctx.save_for_backward(q, q_scale, rstd, *(t for i, t in enumerate(layers) if i % 3 != 2))
        ys = [_product_q8(q, q_scale, w, sc, b, x.dtype) for w, sc, b in zip(*(layers[i::3] for i in range(3)))]
        return (*ys, *out[3:])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        q, q_scale, rstd, *weights = ctx.saved_tensors
        count = len(ctx.bias_dtypes)
        ds = grads[count] if len(grads) > count else None
        need_x, need_res = ctx.needs_input_grad[:2]
        dx = None
        if need_x or need_res:
            dz = None
            # The layers' gradients add up in fp32, and the norm's backward takes the sum as it is.
            for dy, w, sc in zip(grads, weights[::2], weights[1::2]):
                if dy is not None:
                    dz = _input_grad_q8(dy, w, sc, torch.float32, add=dz)
            if dz is None:
                dx = ds
            else:
                dx = binding.msrms_q8_bwd(dz, q, q_scale, rstd, None if ds is None else _flat(ds), dtype=ctx.dtype)
        db = [_bias_grad(grads[i], t) if ctx.needs_input_grad[5 + 3 * i] and grads[i] is not None else None
              for i, t in enumerate(ctx.bias_dtypes)]
        return (dx if need_x else None, dx if need_res else None, None,
                *(g for b in db for g in (None, None, b)))


class MSRMSNormLinearQ8(nn.Module):
    """Residual addition, RMSNorm without weight (Alg. 3; its affine merged into the layers)
    and the ``LinearQ8`` layers behind it. ``forward(x, res)`` returns the layers' outputs and
    s = x + res; ``forward(x)`` the outputs alone (one tensor for a single layer).

    The layers' weights are read and their operators called here, not the layers themselves: what
    only a layer's own call would run (hooks on it, a wrapper, a subclass's forward) is refused.

    To capture forward and backward in a graph, let go of the eager graphs of the same leaves
    first: autograd would wait for the stream that they ran on."""

    def __init__(self, layers, eps=1e-5):
        super().__init__()
        self.layers = nn.ModuleList(layers)
        if not self.layers:
            raise TypeError("layers must be LinearQ8 modules")
        self._check_layers()
        self.eps = float(eps)

    def _check_layers(self):
        for m in self.layers:
            if not isinstance(m, LinearQ8) or type(m).forward is not LinearQ8.forward or "forward" in m.__dict__:
                raise TypeError("layers must be LinearQ8 modules with no forward of their own: it would not run")
            if m._forward_hooks or m._forward_pre_hooks or m._backward_hooks or m._backward_pre_hooks:
                raise RuntimeError("a hook on a layer of MSRMSNormLinearQ8 would not run: put it on the module itself")

    def forward(self, x, res=None):
        self._check_layers()
        flat = [t for m in self.layers for t in (m.weight, m.scale, m.bias)]
        out = _NormLinearQ8.apply(x, res, self.eps, *flat)
        return out[0] if len(out) == 1 else out

    def extra_repr(self):
        return f"eps={self.eps}"


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, rotation):
        ctx.rotation = rotation
        ctx.save_for_backward(positions)
        ctx.set_materialize_grads(False)
        return binding.rope_fwd(_head_rows(q), _head_rows(k), positions, rotation)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        (positions,) = ctx.saved_tensors
        if dq is None:
            return None, None if dk is None else binding.rope_bwd(_head_rows(dk), None, positions, ctx.rotation)[0], None, None
        return (*binding.rope_bwd(_head_rows(dq), _head_rows(dk), positions, ctx.rotation), None, None)


def _head_rows(t):
    """A tensor of heads as the operators take it: copied only if its rows do not lie one behind the other."""
    if t is None:
        return None
    try:
        binding._heads(t, "a tensor")
    except ValueError:
        return t.contiguous()
    return t


def _wide_rows(t):
    """The same for attention, which reads 16 bytes at a time."""
    t = _head_rows(t)
    return t if t.data_ptr() % 16 == 0 and all(s % 8 == 0 for s in t.stride()[:-1]) else t.clone(memory_format=torch.contiguous_format)


def _flat_positions(positions):
    return positions if positions is None or positions.is_contiguous() else positions.contiguous()


class Rope(nn.Module):
    """Rotary positions: forward(q, k, positions) turns both, q [..., heads, dim], k the same with its own
    heads (or None); positions one whole number per row, or [axes, rows]."""

    def __init__(self, rotation):
        super().__init__()
        self.rotation = rotation

    def forward(self, q, k, positions):
        return _Rope.apply(q, k, _flat_positions(positions), self.rotation)

    def extra_repr(self):
        return repr(self.rotation)


class _NormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, rotation, eps, q_gain, k_gain):
        q, k = _head_rows(q), _head_rows(k)
        yq, yk, rstd_q, rstd_k = binding.msrms_rope_fwd(q, k, eps, positions, rotation, q_gain, k_gain)
        ctx.rotation = rotation
        kept = (yq, yk) if q_gain is None else (q, k)
        ctx.save_for_backward(*kept, rstd_q, rstd_k, positions, q_gain, k_gain)
        return yq, yk

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        q, k, rstd_q, rstd_k, positions, q_gain, k_gain = ctx.saved_tensors
        out = binding.msrms_rope_bwd(_head_rows(dq), _head_rows(dk), _head_rows(q), _head_rows(k), rstd_q, rstd_k, positions, ctx.rotation,
                                     q_gain, k_gain)
        return (*out[:2], None, None, None, *(out[2:] if q_gain is not None else (None, None)))


class MSRMSNormRope(nn.Module):
    """RMSNorm of each head (Alg. 3) and the rotation in one pass: forward(q, k, positions) as Rope. ``dim``: the heads'
    width, for a gain per column of q and of k (parameters, fp32 unless ``dtype`` says otherwise); None: no gains."""

    def __init__(self, rotation, eps=1e-5, dim=None, device=None, dtype=torch.float32):
        super().__init__()
        self.rotation, self.eps = rotation, float(eps)
        self.q_gain = None if dim is None else nn.Parameter(torch.ones(dim, device=device, dtype=dtype))
        self.k_gain = None if dim is None else nn.Parameter(torch.ones(dim, device=device, dtype=dtype))

    def forward(self, q, k, positions):
        return _NormRope.apply(q, k, _flat_positions(positions), self.rotation, self.eps, self.q_gain,
                               None if k is None else self.k_gain)

    def extra_repr(self):
        return f"{self.rotation}, eps={self.eps}, gains={self.q_gain is not None}"


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, q_starts, k_starts, k_lens):
        q, k, v = _wide_rows(q), _wide_rows(k), _wide_rows(v)
        o, lse = binding.attention_fwd(q, k, v, causal, scale, q_starts, k_starts, k_lens)
        ctx.how = causal, scale
        ctx.save_for_backward(q, k, v, o, lse, q_starts, k_starts, k_lens)
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, *where = ctx.saved_tensors
        grads = binding.attention_bwd(_wide_rows(do), *(_wide_rows(t) for t in (q, k, v, o)), lse.contiguous(), *ctx.how, *where)
        return (*grads, None, None, None, None, None)


class Attention(nn.Module):
    """softmax(scale q k^T) v (bf16): forward(q, k, v) with q [sequences, rows, heads, dim] and k, v the same with
    their own rows and heads, or packed as [rows, heads, dim] with q_starts / k_starts (int32, sequences + 1);
    k_lens: keys in use of each sequence. Causal: the last query sees the last key. scale: dim ** -0.5 unless given.
    Tensors whose rows do not lie one behind the other ([sequences, heads, rows, dim], the first rows of each of a cache's
    sequences) are copied by every call: a cache lies as [sequences, room, heads, dim] and is given whole, with k_lens."""

    def __init__(self, causal=False, scale=None):
        super().__init__()
        self.causal, self.scale = bool(causal), scale

    def forward(self, q, k, v, q_starts=None, k_starts=None, k_lens=None):
        return _Attention.apply(q, k, v, self.causal, self.scale, q_starts, k_starts, k_lens)

    def extra_repr(self):
        return f"causal={self.causal}, scale={self.scale}"


class _QKVAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, positions, starts, rotation, heads, kv_heads, causal, scale, eps):
        qkv = _wide_rows(qkv)
        q, k, v = qkv.split((heads, kv_heads, kv_heads), -2)
        rstd = (None, None)
        if eps is not None:
            q, k, *rstd = binding.msrms_rope_fwd(q, k, eps, positions, rotation)
        elif rotation.freqs:
            q, k = binding.rope_fwd(q, k, positions, rotation)
        o, lse = binding.attention_fwd(q, k, v, causal, scale, starts, starts)
        ctx.how = rotation, causal, scale, eps
        ctx.save_for_backward(q, k, v, o, lse, positions, starts, *rstd)
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, positions, starts, rstd_q, rstd_k = ctx.saved_tensors
        rotation, causal, scale, eps = ctx.how
        heads, kv_heads = q.shape[-2], k.shape[-2]
        d = torch.empty((*q.shape[:-2], heads + 2 * kv_heads, q.shape[-1]), dtype=q.dtype, device=q.device)
        if starts is not None:
            d.zero_()   # rows of no sequence
        dq, dk, dv = d.split((heads, kv_heads, kv_heads), -2)
        q, k, v, o = (_wide_rows(t) for t in (q, k, v, o))
        # dq and dk are rounded to the type here, and again where they are turned back in place: between the two kernels
        # fp32 would take its own tensors, written and read once
        binding.attention_bwd(_wide_rows(do), q, k, v, o, lse.contiguous(), causal, scale, starts, starts, dq=dq, dk=dk, dv=dv)
        if eps is not None:
            binding.msrms_rope_bwd(dq, dk, q, k, rstd_q, rstd_k, positions, rotation, q_out=dq, k_out=dk)
        elif rotation.freqs:
            binding.rope_bwd(dq, dk, positions, rotation, q_out=dq, k_out=dk)
        return d, None, None, None, None, None, None, None, None


class QKVAttention(nn.Module):
    """Rotation and attention on the output of a block's fused projection: forward(qkv, positions) with qkv
    [sequences, rows, heads + 2 kv_heads, dim] (queries, keys, values) gives [sequences, rows, heads, dim]; packed as
    [rows, ..] with ``starts`` (int32, sequences + 1; rows behind the last one may hold anything, their output and gradient are zeros).
    ``eps``: MS-RMSNorm of each query and key head in front of the
    rotation (without gains). One node: keeps the turned queries and keys, the values as they lie in qkv,
    the output and one fp32 value per row and head (with the norm one more per query and key head); the gradient comes as one
    tensor. To capture forward and backward of this or the modules above in a graph, let go of the eager graphs of the
    same leaves first."""

    def __init__(self, heads, kv_heads, dim, rotation, causal=True, scale=None, eps=None):
        super().__init__()
        if heads % kv_heads:
            raise ValueError("kv_heads must divide heads")
        if 2 * len(rotation.freqs) > dim:
            raise ValueError("the rotation has more columns than a head")
        self.heads, self.kv_heads, self.dim, self.rotation = heads, kv_heads, dim, rotation
        self.causal, self.scale, self.eps = bool(causal), scale, None if eps is None else float(eps)

    def forward(self, qkv, positions, starts=None):
        if qkv.shape[-2:] != (self.heads + 2 * self.kv_heads, self.dim):
            raise ValueError(f"qkv must be [..., {self.heads + 2 * self.kv_heads}, {self.dim}]")
        return _QKVAttention.apply(qkv, _flat_positions(positions), starts, self.rotation, self.heads, self.kv_heads, self.causal,
                                   self.scale, self.eps)

    def extra_repr(self):
        return (f"heads={self.heads}, kv_heads={self.kv_heads}, dim={self.dim}, {self.rotation}, causal={self.causal}, "
                f"eps={self.eps}")


@torch.no_grad()
def merge_affine_into_linear(linear, alpha, beta=None):
    """In place: W <- W diag(alpha); b <- W beta + b (Sec. 5.2). The products are formed
    in float64 and rounded once to the layer's dtype. A bias is created if beta is
    given and the layer had none."""
    W = linear.weight
    if W.shape[1] != alpha.numel():
        raise ValueError("alpha must have one entry per input feature of the linear layer")
    W64 = W.double()
    a64 = alpha.detach().to(W.device, torch.float64).reshape(-1)
    if beta is not None:
        b_add = W64 @ beta.detach().to(W.device, torch.float64).reshape(-1)
        if linear.bias is None:
            linear.bias = nn.Parameter(b_add.to(W.dtype))
        else:
            linear.bias.copy_((linear.bias.double() + b_add).to(linear.bias.dtype))
    W.copy_((W64 * a64[None, :]).to(W.dtype))
    return linear


@torch.no_grad()
def merge_norm_into_linears(norm, linears):
    """Fold the affine of ``norm`` (a torch LayerNorm or RMSNorm with elementwise
    affine) into every linear layer that consumes its output, and return the
    parameter-free MS norm that replaces it. Requires normalization over one
    (the last) dimension."""
    if not isinstance(norm, (nn.LayerNorm, nn.RMSNorm)):
        raise TypeError("norm must be torch.nn.LayerNorm or torch.nn.RMSNorm")
    shape = tuple(norm.normalized_shape)
    if len(shape) != 1:
        raise ValueError("only normalization over the last dimension is supported")
    alpha = norm.weight if norm.weight is not None else torch.ones(shape[0])
    if isinstance(norm, nn.LayerNorm):
        beta = norm.bias
        ms = MSLayerNorm(norm.eps)
    elif isinstance(norm, nn.RMSNorm):
        beta = None
        eps = norm.eps if norm.eps is not None else torch.finfo(torch.float32).eps
        ms = MSRMSNorm(eps)
    for lin in linears:
        merge_affine_into_linear(lin, alpha, beta)
    return ms
