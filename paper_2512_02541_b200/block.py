"""What stands around the attention of a block: rotary positions with the norm of the heads, and the residual stream with its norms
and gate, forward and backward.  PyTorch is used for device memory and streams only: the calls enqueue the library's kernels on
the current stream of the inputs' device and are not recorded by autograd, whatever requires a gradient (results carry no graph);
gradients are computed by the ``backward`` methods.

The checks are written to be cheap: a call on few tokens is as long as the host takes for it (a frame's rotary positions: 24 us with
checks in general form and ctypes structures, 15 as they are, of which the kernel runs for 8).
"""

import ctypes
import operator
from collections import namedtuple

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.AVGGT_TYPE_BF16, torch.float16: B.AVGGT_TYPE_FP16, torch.float32: B.AVGGT_TYPE_FP32}
_F32 = torch.float32
_contiguous = torch.contiguous_format
# what torch.cuda.current_device() and torch.cuda.current_stream(index).cuda_stream give, without what they do on the way (there is a
# CUDA tensor in hand where these are called); themselves where this torch does not have the short forms
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)

RotaryGrads = namedtuple("RotaryGrads", "dq dk dv q_weight q_bias k_weight k_bias")
ResidualGrads = namedtuple("ResidualGrads", "dx dy weight bias gate post_weight post_bias")


def token_positions(params, time=False, first_frame=0, device="cuda"):
    """int32 [N*L, 2 or 3]: the positions of a problem's tokens as VGGT counts them, row + 1 and column + 1 of a patch token in its
    frame's grid, zeros for the special tokens; with ``time`` the frame's number, from ``first_frame`` on, in front of them."""
    t = torch.arange(params.n_frames * params.tokens_per_frame, device=device)
    slot = t % params.tokens_per_frame - params.n_special
    patch = slot >= 0
    axes = [torch.where(patch, slot // params.grid_w + 1, 0), torch.where(patch, slot % params.grid_w + 1, 0)]
    if time:
        axes.insert(0, t // params.tokens_per_frame + first_frame)
    return torch.stack(axes, 1).to(torch.int32)


def _call(name, index, *args):
    """The entry point, with device ``index`` current."""
    if _current_device() == index:
        code = B.packed_entry(name)(*args)
    else:
        with torch.cuda.device(index):
            code = B.packed_entry(name)(*args)
    if code:
        raise B.AvggtError(code, name)


def _workspace(query, params, index):
    """A new workspace of the size that the entry point ``query`` gives: of each call its own, so that calls on several streams, or
    captured into several graphs, share none."""
    size = ctypes.c_size_t()
    _call(query, index, params, ctypes.byref(size))
    return torch.empty((size.value,), dtype=torch.uint8, device=index)


def _first(name, t, dims):
    """The tensor that a call's sizes are taken from -> its type, its device's index and AVGGT_TYPE_*."""
    kind = _TYPES.get(t.dtype)
    if not t.is_cuda or kind is None or t.dim() != dims:
        raise ValueError(f"{name}: expected a CUDA tensor of bfloat16, float16 or float32 with {dims} dimensions")
    return t.dtype, t.get_device(), kind


def _refuse(name, shape, dtype, index):
    raise ValueError(f"{name}: expected a {dtype} tensor of shape {tuple(shape)} on cuda:{index} whose last dimension is contiguous")


def _heads(name, t, shape, dtype, index):
    """A checked [n_tokens, heads, head_dim] tensor as the library takes it."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        _refuse(name, shape, dtype, index)
    token, head, last = t.stride()
    if last != 1 and shape[2] > 1:
        _refuse(name, shape, dtype, index)
    return B.PACKED_HEADS.pack(t.data_ptr(), token, head)


def _rows(name, t, shape, dtype, index):
    """A checked [n_tokens, channels] tensor as the library takes it."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        _refuse(name, shape, dtype, index)
    row, last = t.stride()
    if last != 1 and shape[1] > 1:
        _refuse(name, shape, dtype, index)
    return B.PACKED_ROWS.pack(t.data_ptr(), row)


def _param(name, t, shape, index):
    """The address of a checked weight, bias or gate, or None."""
    if t is None:
        return None
    if t.dtype is not _F32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous float32 tensor of shape {tuple(shape)} on cuda:{index}")
    return t.data_ptr()


def _address(t):
    return None if t is None else t.data_ptr()


class AxialRotary:
    """Rotary positions on one to three axes behind the norm of each head of Q and K (``avggt_rotary``).

    ``pairs``: the pairs of elements that each axis turns.  Each axis has a block of the head and a ladder of frequencies
    theta^(-j / pairs) of its own, or, with ``shared_ladder``, one block and one ladder for all axes.  ``adjacent``: pairs are
    neighbouring elements instead of a block's two halves.  ``norm``: AVGGT_NORM_* of the heads.
    """

    def __init__(self, head_dim, pairs, theta=100.0, *, shared_ladder=False, adjacent=False, norm=B.AVGGT_NORM_NONE, eps=1e-5):
        pairs = tuple(int(n) for n in pairs)
        if not 1 <= len(pairs) <= 3:
            raise ValueError("expected pairs for one to three axes")
        self.head_dim, self.pairs, self.norm, self.eps, self.theta = head_dim, pairs, norm, eps, theta
        flags = (B.AVGGT_ROTARY_SHARED_LADDER if shared_ladder else 0) | (B.AVGGT_ROTARY_ADJACENT if adjacent else 0)
        # the parameters' fields behind the sizes of a call, of each type
        self._rest = [B.PACKED_ROTARY_REST.pack(head_dim, len(pairs), *pairs, *(0,) * (3 - len(pairs)), kind, norm, eps, flags)
                      for kind in range(len(_TYPES))]

    def params(self, n_tokens, heads_q, heads_k, dtype):
        """The C ABI's parameters of a call."""
        return B.AvggtRotaryParams.from_buffer_copy(B.PACKED_ROTARY_SIZES.pack(n_tokens, self.theta, heads_q, heads_k) + self._rest[_TYPES[dtype]])

    def _sizes(self, q, k, v, positions, names):
        """Of the tensors of either direction -> type, index of the index, packed parameters, shapes of Q and of K and V."""
        if q is None and k is None:
            raise ValueError(f"expected {names[0]} or {names[1]}")
        dtype, index, kind = _first(names[0], q, 3) if q is not None else _first(names[1], k, 3)
        T, heads, _ = (q if q is not None else k).shape
        heads_q = heads_k = heads
        if q is not None and (k is not None or v is not None):
            like = k if k is not None else v
            if like.dim() != 3:
                _refuse(names[1] if k is not None else names[2], (T, heads, self.head_dim), dtype, index)
            heads_k = like.shape[1]
        axes = len(self.pairs)
        if positions.dtype is not torch.int32 or positions.shape != (T, axes) or positions.get_device() != index or not positions.is_contiguous():
            raise ValueError(f"positions: expected a contiguous int32 tensor of shape {(T, axes)} on cuda:{index}")
        d = self.head_dim
        return dtype, index, B.PACKED_ROTARY_SIZES.pack(T, self.theta, heads_q, heads_k) + self._rest[kind], (T, heads_q, d), (T, heads_k, d)

    @staticmethod
    def _output(name, given, like, shape, dtype, index):
        """-> the tensor that a result goes to, new where none is given, and its packed form."""
        if like is None:
            return None, None
        if given is not None:
            return given, _heads(name, given, shape, dtype, index)
        t = torch.empty_like(like, memory_format=_contiguous)
        return t, B.PACKED_HEADS.pack(t.data_ptr(), shape[1] * shape[2], shape[2])

    def forward(self, q, k, positions, v=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None, out=None):
        """-> (Q, K, V), contiguous unless ``out`` = (Q, K, V) says where they go (None: a new tensor; an input itself: in place).

        q, k, v: [n_tokens, heads, head_dim], strided as a projection leaves them; any but the last of q and k may be None.  positions:
        int32 [n_tokens, axes].  Weights and biases of the norms: float32 [head_dim], or None.
        """
        dtype, index, params, shape_q, shape_k = self._sizes(q, k, v, positions, ("q", "k", "v"))
        row = (self.head_dim,)
        out_q, out_k, out_v = (None, None, None) if out is None else out
        heads = (None if q is None else _heads("q", q, shape_q, dtype, index), None if k is None else _heads("k", k, shape_k, dtype, index),
                 None if v is None else _heads("v", v, shape_k, dtype, index))
        rows = (_param("q_weight", q_weight, row, index), _param("q_bias", q_bias, row, index), _param("k_weight", k_weight, row, index),
                _param("k_bias", k_bias, row, index))
        Q, packed_q = self._output("out[0]", out_q, q, shape_q, dtype, index)
        K, packed_k = self._output("out[1]", out_k, k, shape_k, dtype, index)
        V, packed_v = self._output("out[2]", out_v, v, shape_k, dtype, index)
        _call("avggt_rotary", index, params, positions.data_ptr(), *heads, *rows, packed_q, packed_k, packed_v, _stream(index))
        return Q, K, V

    __call__ = forward

    def backward(self, dq, dk, positions, q=None, k=None, dv=None, q_weight=None, q_bias=None, k_weight=None, k_bias=None, out=None,
                 parameter_grads=True):
        """Gradients of ``forward``'s outputs -> RotaryGrads of its inputs (into ``out`` = (dq, dk, dv) where given) and of the weights
        and biases that are given (float32; None of the others, and of all without ``parameter_grads``).  q, k: the inputs of
        the forward call, needed where there is a norm."""
        dtype, index, params, shape_q, shape_k = self._sizes(dq, dk, dv, positions, ("dq", "dk", "dv"))
        normed = self.norm != B.AVGGT_NORM_NONE
        row = (self.head_dim,)
        out_q, out_k, out_v = (None, None, None) if out is None else out
        heads = (None if dq is None else _heads("dq", dq, shape_q, dtype, index), None if dk is None else _heads("dk", dk, shape_k, dtype, index),
                 None if dv is None else _heads("dv", dv, shape_k, dtype, index))
        inputs = [None, None]
        for i, (name, x, grad, shape) in enumerate((("q", q, dq, shape_q), ("k", k, dk, shape_k))):
            if normed and grad is not None:
                if x is None:
                    raise ValueError(f"{name}: the gradient through the norm needs the forward call's input")
                inputs[i] = _heads(name, x, shape, dtype, index)
        weight_q, weight_k = _param("q_weight", q_weight, row, index), _param("k_weight", k_weight, row, index)
        _param("q_bias", q_bias, row, index)
        _param("k_bias", k_bias, row, index)
        gq, packed_q = self._output("out[0]", out_q, dq, shape_q, dtype, index)
        gk, packed_k = self._output("out[1]", out_k, dk, shape_k, dtype, index)
        gv, packed_v = self._output("out[2]", out_v, dv, shape_k, dtype, index)
        rows = [torch.empty_like(t) if t is not None and grad is not None and parameter_grads else None
                for t, grad in ((q_weight, dq), (q_bias, dq), (k_weight, dk), (k_bias, dk))]
        ws, ws_bytes = None, 0
        if normed:
            ws = _workspace("avggt_rotary_workspace_bytes", params, index)
            ws_bytes = ws.numel()
        _call("avggt_rotary_backward", index, params, positions.data_ptr(), *heads, *inputs, weight_q, weight_k, packed_q, packed_k,
              packed_v, *map(_address, rows), _address(ws), ws_bytes, _stream(index))
        return RotaryGrads(gq, gk, gv, *rows)


class ResidualNorm:
    """The residual stream between two branches of a block (``avggt_residual_norm``):

        r = residual_scale * x + gate * post_norm(y),     h = norm(r) * weight + bias

    ``norm`` and ``post_norm``: AVGGT_NORM_* in front of the next branch and behind the last one.  ``one_plus_weight``: 1 + weight
    multiplies the norm.  A weight, bias or gate of shape [groups, channels] has a row for every ``tokens_per_group`` tokens; weight
    and bias, where both are given, have the same shape.
    """

    def __init__(self, channels, *, norm=B.AVGGT_NORM_LAYER, eps=1e-5, post_norm=B.AVGGT_NORM_NONE, post_eps=1e-5, residual_scale=1.0,
                 one_plus_weight=False, tokens_per_group=None):
        if tokens_per_group is not None:
            try:
                tokens_per_group = operator.index(tokens_per_group)
            except TypeError:
                raise ValueError(f"tokens_per_group: expected a whole number, not {tokens_per_group!r}") from None
        self.channels, self.norm, self.eps, self.post_norm, self.post_eps = channels, norm, eps, post_norm, post_eps
        self.residual_scale, self.one_plus_weight, self.tokens_per_group = residual_scale, one_plus_weight, tokens_per_group

    def _params(self, T, index, residual_kind, branch_kind, weight, bias, gate, post_weight, post_bias):
        """-> the fields of the C ABI's parameters, and the addresses of the checked weight, bias, gate, post_weight and post_bias."""
        C, per_group = self.channels, self.tokens_per_group
        flags = B.AVGGT_RESIDUAL_ONE_PLUS_WEIGHT if self.one_plus_weight else 0
        shape_w = shape_g = row = (C,)
        like = weight if weight is not None else bias
        grouped_w, grouped_g = like is not None and like.dim() == 2, gate is not None and gate.dim() == 2
        if grouped_w or grouped_g:
            if per_group is None or per_group < 1:
                raise ValueError("a weight, bias or gate for each group needs tokens_per_group of at least 1")
            groups = (-(-T // per_group), C)
            if grouped_w:
                flags |= B.AVGGT_RESIDUAL_WEIGHT_GROUPED
                shape_w = groups
            if grouped_g:
                flags |= B.AVGGT_RESIDUAL_GATE_GROUPED
                shape_g = groups
        fields = (T, per_group or 1, C, residual_kind, branch_kind, self.norm, self.post_norm, self.eps, self.post_eps, self.residual_scale, flags)
        return (fields, _param("weight", weight, shape_w, index), _param("bias", bias, shape_w, index), _param("gate", gate, shape_g, index),
                _param("post_weight", post_weight, row, index), _param("post_bias", post_bias, row, index))

    def forward(self, x, y=None, *, weight=None, bias=None, gate=None, post_weight=None, post_bias=None, branch_dtype=None, out_r=None,
                out_h=None):
        """-> (r, h).  x, y: [n_tokens, channels], rows strided as they are.  Without ``y`` (the first norm of a model) r is
        residual_scale * x, which is written only where ``out_r`` asks for it (x itself is returned where the scale is 1).  h has y's
        type (without y: ``branch_dtype``, or x's); h is None where ``norm`` is AVGGT_NORM_NONE.  ``out_r`` may be x, ``out_h`` may be y."""
        dtype, index, kind = _first("x", x, 2)
        shape = (x.shape[0], self.channels)
        rows_x = _rows("x", x, shape, dtype, index)
        branch, branch_kind, rows_y = dtype, kind, None
        if y is not None:
            branch, _, branch_kind = _first("y", y, 2)
            rows_y = _rows("y", y, shape, branch, index)
        elif branch_dtype is not None or out_h is not None:
            branch = branch_dtype if branch_dtype is not None else out_h.dtype
            branch_kind = _TYPES.get(branch)
            if branch_kind is None:
                raise ValueError("expected a branch of bfloat16, float16 or float32")
        fields, *params = self._params(shape[0], index, kind, branch_kind, weight, bias, gate, post_weight, post_bias)
        r, h, rows_r, rows_h = out_r, out_h, None, None
        if r is not None:
            rows_r = _rows("out_r", r, shape, dtype, index)
        elif y is not None or self.residual_scale != 1.0:
            r = torch.empty_like(x, memory_format=_contiguous)
            rows_r = B.PACKED_ROWS.pack(r.data_ptr(), self.channels)
        if h is not None:
            rows_h = _rows("out_h", h, shape, branch, index)
        elif self.norm != B.AVGGT_NORM_NONE:
            h = torch.empty_like(x if y is None else y, dtype=None if y is not None else branch, memory_format=_contiguous)
            rows_h = B.PACKED_ROWS.pack(h.data_ptr(), self.channels)
        if r is None and h is None:
            return x, None
        _call("avggt_residual_norm", index, B.PACKED_RESIDUAL.pack(*fields), rows_x, rows_y, *params, rows_r, rows_h,
              _stream(index))
        return (x if r is None else r), h

    __call__ = forward

    def backward(self, dh, dr, r, y=None, *, weight=None, bias=None, gate=None, post_weight=None, post_bias=None, out_dx=None, out_dy=None,
                 parameter_grads=True):
        """Gradients of h and of r (either may be None) -> ResidualGrads of x, of y (where it is given) and of the parameters that are
        given (float32; None of the others, and of all without ``parameter_grads``).  r: ``forward``'s.  ``out_dx`` may be dr or
        r, ``out_dy`` may be dh or y."""
        if dh is None and dr is None:
            raise ValueError("expected the gradient of h or of r")
        if dh is not None and r is None:
            raise ValueError("r: the gradient through the norm needs it")
        if y is None and out_dy is not None:
            raise ValueError("out_dy: there is no branch")
        like, name = (dr, "dr") if dr is not None else (r, "r")
        dtype, index, kind = _first(name, like, 2)
        branch, _, branch_kind = (dtype, index, kind) if dh is None and y is None else _first("dh", dh, 2) if dh is not None else _first("y", y, 2)
        shape = (like.shape[0], self.channels)
        rows = lambda name, t, dtype: None if t is None else _rows(name, t, shape, dtype, index)
        dx = out_dx if out_dx is not None else torch.empty_like(like, memory_format=_contiguous)
        dy = out_dy if out_dy is not None or y is None else torch.empty_like(y, memory_format=_contiguous)
        arrays = (rows("dh", dh, branch), rows("dr", dr, dtype), rows("r", r, dtype), rows("y", y, branch))
        fields, address_w, _, address_g, address_pw, address_pb = self._params(shape[0], index, kind, branch_kind, weight, bias, gate, post_weight,
                                                                               post_bias)
        packed = B.PACKED_RESIDUAL.pack(*fields)
        through_norm, has_branch = dh is not None, y is not None
        grads = [torch.empty_like(t) if t is not None and there and parameter_grads else None
                 for t, there in ((weight, through_norm), (bias, through_norm), (gate, has_branch), (post_weight, has_branch),
                                  (post_bias, has_branch))]
        ws, ws_bytes = None, 0
        if any(t is not None for t in grads):
            ws = _workspace("avggt_residual_workspace_bytes", packed, index)
            ws_bytes = ws.numel()
        _call("avggt_residual_norm_backward", index, packed, *arrays, address_w, address_g, address_pw, address_pb,
              rows("out_dx", dx, dtype), rows("out_dy", dy, branch), *map(_address, grads), _address(ws), ws_bytes,
              _stream(index))
        return ResidualGrads(dx, dy, *grads)
