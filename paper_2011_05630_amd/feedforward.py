"""The feed-forward half of a transformer block on libdlf: a linear layer with bias, activation and residual in one kernel,
a gated pair of projections in one kernel, the block of the two, and their gradients.

The objects hold the caller's weight tensors (no copies: change their values and the next call sees it; a tensor whose shape,
type, row distance or device has changed is refused).  PyTorch provides device memory and streams only.  Every call runs on
the current stream of the weights' device, asynchronously; outputs, saved tensors and workspaces come from PyTorch's allocator,
so calls may be captured into a graph.  A tensor that another stream wrote or will overwrite is ordered by the caller, as for
any kernel.

Automatic differentiation does not see the calls, so an operand that requires a gradient (while gradients are recorded) or carries a
tangent is refused: call under torch.no_grad(), or inside a torch.autograd.Function's forward and backward, and take the gradients from
`run_saved` and `backward`.

Tensors are fp16 or bf16, all of one type, with rows of consecutive elements at any alignment and any distance below
2^24 elements (of a single row it says nothing); biases and their gradients fp32.  Inputs may have any number of leading dimensions
that lie at one row distance.
"""
import torch

from . import binding as B

_TYPES = (torch.float16, torch.bfloat16)


def _native():
    B.lib()                     # a missing library says so itself
    try:
        from . import _dlf_torch
    except ImportError as e:
        raise RuntimeError("_dlf_torch.so is not built, or not for this PyTorch: run `python -m paper_2011_05630_amd.build` first (%s)" % e) from e
    if _dlf_torch.built_with != "built with PyTorch " + torch.__version__:
        raise RuntimeError("_dlf_torch.so is %s, this is %s: run `python -m paper_2011_05630_amd.build` again" % (_dlf_torch.built_with, torch.__version__))
    return _dlf_torch


def _stream(index):
    return torch._C._cuda_getCurrentRawStream(index)


def _need(ok, msg, *a):
    if not ok:
        raise ValueError(msg % a if a else msg)


_GRADIENTS = ("x", "weight", "bias")


def _wanted(need):
    """Which of _GRADIENTS `need` names, which is some of them, or one."""
    if need is _GRADIENTS:
        return True, True, True
    need = (need,) if isinstance(need, str) else tuple(need)
    for n in need:
        _need(n in _GRADIENTS, "need: some of %s expected, not %r", ", ".join(_GRADIENTS), n)
    return tuple(g in need for g in _GRADIENTS)


def _weight(t, name):
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype in _TYPES and not t.is_neg(), "%s: a 2-dimensional fp16 or bf16 tensor on the GPU expected", name)
    _need(t.shape[0] > 0 and t.shape[1] > 0, "%s: empty", name)
    _stride(t, name)
    return t


def _bias(t, n, w, name):
    _need(t is None or (isinstance(t, torch.Tensor) and t.device == w.device and t.dtype == torch.float32 and tuple(t.shape) == (n,) and t.is_contiguous() and not t.is_neg()),
          "%s: a contiguous fp32 tensor of %d elements on the weight's device expected", name, n)
    return t


def _stride(t, name):
    """Distance of the rows of a 2-dimensional tensor whose rows are consecutive elements."""
    _need(t.shape[1] == 1 or t.stride(1) == 1, "%s: a row's elements have to lie next to each other", name)
    s = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    _need(s >= t.shape[1], "%s: rows overlap", name)
    return s


class _Operator:
    """What the operators share: the weights' type, device and sizes, and the native operator that holds them."""

    def _setup(self, gated, act, weights, biases):
        if act not in B.FF_ACT:
            raise ValueError("act: one of %s expected" % ", ".join(sorted(B.FF_ACT)))
        w = weights[0]
        self.act, self.dtype, self.device = act, w.dtype, w.device
        self.out_features, self.in_features = w.shape
        self._index = w.get_device()
        op = _native().Op(gated, B.FF_ACT[act], *weights, *biases, _stride(w, "weight"))
        self._forward, self._backward = op.forward, op.backward
        self._fixed = frozenset(self.__dict__)

    # The native operator holds what it was made of, and would not see another tensor in its place here.
    def __setattr__(self, name, value):
        self._refuse_fixed(name)
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        self._refuse_fixed(name)
        object.__delattr__(self, name)

    def _refuse_fixed(self, name):
        if name in self.__dict__.get("_fixed", ()):
            raise AttributeError("%s: fixed when the operator was made; change the tensor's values, or make another operator" % name)


class Linear(_Operator):
    """y = act(x weight^T + bias) + residual.  weight [out, in] fp16 or bf16, bias fp32 [out] or None."""

    def __init__(self, weight, bias=None, act="none"):
        self.weight = _weight(weight, "weight")
        self.bias = _bias(bias, weight.shape[0], weight, "bias")
        self._setup(False, act, (weight, None), (bias, None))

    def run(self, x, residual=None, out=None):
        """-> y [..., out]; written to `out` if given (which may be the residual, and is refused on x or a weight)."""
        return self._forward(x, residual, out, False, _stream(self._index))

    def run_saved(self, x, residual=None, out=None):
        """-> (y, saved): the pre-activations that `backward` needs, fp32 [rows, out]; None without an activation."""
        return self._forward(x, residual, out, True, _stream(self._index))

    def backward(self, dy, x, saved, need=_GRADIENTS):
        """Gradients for dy, the gradient of y: -> (dx, dweight, dbias), None for what `need` leaves out or the layer lacks.
        x and saved are those of the forward call.  The gradient of its residual is dy."""
        return self._backward(dy, x, saved, *_wanted(need), _stream(self._index))


class GatedLinear(_Operator):
    """h = act(x w_gate^T + b_gate) * (x w_up^T + b_up).  w_gate, w_up [out, in], of one type and row distance (two halves of one
    tensor among others), biases fp32 [out] or None."""

    def __init__(self, w_gate, w_up, b_gate=None, b_up=None, act="silu"):
        self.w_gate, self.w_up = _weight(w_gate, "w_gate"), _weight(w_up, "w_up")
        _need(w_up.shape == w_gate.shape and w_up.dtype == w_gate.dtype and w_up.device == w_gate.device and
              _stride(w_up, "w_up") == _stride(w_gate, "w_gate"), "w_up: shape, type, device and row distance of w_gate expected")
        self.b_gate, self.b_up = (_bias(b, w_gate.shape[0], w_gate, n) for b, n in ((b_gate, "b_gate"), (b_up, "b_up")))
        self._setup(True, act, (w_gate, w_up), (b_gate, b_up))

    def run(self, x, out=None):
        """-> h [..., out]; written to `out` if given (which is refused on x or a weight)."""
        return self._forward(x, None, out, False, _stream(self._index))

    def run_saved(self, x, out=None):
        """-> (h, saved): both projections' results, which `backward` needs, fp32 [2, rows, out]."""
        return self._forward(x, None, out, True, _stream(self._index))

    def backward(self, dh, x, saved, need=_GRADIENTS):
        """Gradients for dh, the gradient of h: -> (dx, dw_gate, dw_up, db_gate, db_up), None for what `need` leaves out or the
        layer lacks.  x and saved are those of the forward call."""
        return self._backward(dh, x, saved, *_wanted(need), _stream(self._index))


class FeedForward:
    """The block y = down(gated(x)) + residual: two kernels forward.  h, between the two products, and its gradient, between the two backward
    calls, are tensors of the weights' type, with its rounding and its range (fp16: infinite above 65504, zero below 2^-25)."""

    def __init__(self, gated, down):
        _need(isinstance(gated, GatedLinear) and isinstance(down, Linear), "a GatedLinear and a Linear expected")
        _need(down.in_features == gated.out_features and down.dtype == gated.dtype and down.device == gated.device,
              "down: %d input features of type %s on %s expected", gated.out_features, gated.dtype, gated.device)
        self.gated, self.down = gated, down

    def run(self, x, residual=None, out=None):
        """-> y [..., out]; `out` may be x itself where x is the residual."""
        return self.down.run(self.gated.run(x), residual, out)

    def run_saved(self, x, residual=None, out=None):
        """-> (y, saved): what `backward` needs beside x.  `out` may be x itself where x is the residual, for a caller that
        keeps x's values elsewhere for `backward`."""
        h, saved_g = self.gated.run_saved(x)
        y, saved_d = self.down.run_saved(h, residual, out)
        return y, (h, saved_g, saved_d)

    def backward(self, dy, x, saved, need=_GRADIENTS):
        """-> (dx, (dw_gate, dw_up, db_gate, db_up), (dw_down, db_down)).  dx is the gradient through the products; where x
        was the residual too, dy is added to it by the caller."""
        need = tuple(g for g, w in zip(_GRADIENTS, _wanted(need)) if w)
        h, saved_g, saved_d = saved
        dh, dw, db = self.down.backward(dy, h, saved_d, need + ("x",))
        g = self.gated.backward(dh, x, saved_g, need)
        return g[0], g[1:], (dw, db)
