"""The feed-forward half of a transformer block on libdlf: a linear layer with bias, activation and residual in one kernel,
a gated pair of projections in one kernel, the block of the two, and their gradients.

The objects hold the caller's weight tensors (no copies: change them in place and the next call sees it).  PyTorch provides
device memory and streams only.  Every call runs on the current stream of the weights' device, asynchronously; outputs,
saved tensors and workspaces come from PyTorch's allocator, so calls may be captured into a graph.  A tensor that another
stream wrote or will overwrite is ordered by the caller, as for any kernel.

Tensors are fp16 or bf16, all of one type, with rows of consecutive elements at any distance and alignment; biases and
their gradients fp32.  Inputs may have any number of leading dimensions that lie at one row distance.
"""
import torch

from . import binding as B

_TYPE = {torch.float16: "fp16", torch.bfloat16: "bf16"}


def _need(ok, msg, *a):
    if not ok:
        raise ValueError(msg % a if a else msg)


def _weight(t, name):
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype in _TYPE, "%s: a 2-dimensional fp16 or bf16 tensor on the GPU expected", name)
    _need(t.shape[0] > 0 and t.shape[1] > 0, "%s: empty", name)
    _stride(t, name)
    return t


def _bias(t, n, w, name):
    _need(t is None or (isinstance(t, torch.Tensor) and t.device == w.device and t.dtype == torch.float32 and tuple(t.shape) == (n,) and t.is_contiguous()),
          "%s: a contiguous fp32 tensor of %d elements on the weight's device expected", name, n)
    return t


def _stride(t, name):
    """Distance of the rows of a 2-dimensional tensor whose rows are consecutive elements."""
    _need(t.shape[1] == 1 or t.stride(1) == 1, "%s: a row's elements have to lie next to each other", name)
    s = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    _need(s >= t.shape[1], "%s: rows overlap", name)
    return s


class _Operator:
    """What the operators share: the weights' type, device and sizes, views of the operands as rows, the call itself."""

    def _setup(self, w, act):
        if act not in B.FF_ACT:
            raise ValueError("act: one of %s expected" % ", ".join(sorted(B.FF_ACT)))
        self.act, self.dtype, self.device = act, w.dtype, w.device
        self.out_features, self.in_features = w.shape
        self._index, self._w_stride = w.get_device(), _stride(w, "weight")
        self._calls = {}        # descriptions by call, rows and strides, with the workspace they ask for

    def _rows(self, t, width, name, rows=None):
        """t as rows, and their distance."""
        if not isinstance(t, torch.Tensor) or t.dtype is not self.dtype or t.get_device() != self._index or t.dim() < 1 or t.shape[-1] != width:
            raise ValueError("%s: a %s tensor [..., %d] on %s expected" % (name, self.dtype, width, self.device))
        if t.dim() != 2:
            try:
                t = t.view(-1, width)
            except RuntimeError:
                raise ValueError("%s: its rows do not lie at one distance" % name) from None
        m, (s, one) = t.shape[0], t.stride()
        if rows is not None and m != rows:
            raise ValueError("%s: %d rows expected" % (name, rows))
        if one != 1 and width != 1:
            raise ValueError("%s: a row's elements have to lie next to each other" % name)
        if m <= 1:
            s = width
        elif s < width:
            raise ValueError("%s: rows overlap" % name)
        return t, s

    def _out(self, out, shape, rows):
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
            return out, out, self.out_features
        _need(out.shape == shape, "out: shape %s expected", tuple(shape))
        return (out,) + self._rows(out, self.out_features, "out", rows)

    def _saved(self, saved, shape):
        _need(isinstance(saved, torch.Tensor) and saved.dtype == torch.float32 and saved.device == self.device and tuple(saved.shape) == shape and
              saved.is_contiguous(), "saved: the tensor that the forward call returned, fp32 %s, expected", shape)
        return saved

    def _call(self, name, rows, strides, *tensors):
        """strides: of x, y, residual and dy."""
        key = (name, rows, strides)
        call = self._calls.get(key)
        if call is None:
            xs, ys, rs, ds = strides
            desc = B.dlf_ff_desc(_TYPE[self.dtype], self.act, rows, self.in_features, self.out_features, xs, self._w_stride, ys, rs, ds)
            if len(self._calls) >= 1024:
                self._calls.clear()
            call = self._calls[key] = (getattr(B, name), desc, B._ff_workspace(name, desc))
        f, desc, need = call
        ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        ptr = [None if t is None else t.data_ptr() for t in tensors]
        ptr.append(None if ws is None else ws.data_ptr())
        if torch.cuda.current_device() == self._index:
            f(desc, *ptr, need, torch._C._cuda_getCurrentRawStream(self._index))
        else:
            with torch.cuda.device(self._index):
                f(desc, *ptr, need, torch._C._cuda_getCurrentRawStream(self._index))


class Linear(_Operator):
    """y = act(x weight^T + bias) + residual.  weight [out, in] fp16 or bf16, bias fp32 [out] or None."""

    def __init__(self, weight, bias=None, act="none"):
        self.weight = _weight(weight, "weight")
        self._setup(weight, act)
        self.bias = _bias(bias, self.out_features, weight, "bias")

    def _forward(self, x, residual, out, save):
        x2, xs = self._rows(x, self.in_features, "x")
        rows = x2.shape[0]
        shape = x.shape[:-1] + (self.out_features,)
        rs = 0
        if residual is not None:
            _need(residual.shape == shape, "residual: shape %s expected", tuple(shape))
            residual, rs = self._rows(residual, self.out_features, "residual", rows)
        out, o2, ys = self._out(out, shape, rows)
        saved = torch.empty((rows, self.out_features), dtype=torch.float32, device=self.device) if save and self.act != "none" else None
        self._call("dlf_linear", rows, (xs, ys, rs, 0), x2, self.weight, self.bias, residual, o2, saved)
        return out, saved

    def run(self, x, residual=None, out=None):
        """-> y [..., out]; written to `out` if given (which may be the residual)."""
        return self._forward(x, residual, out, False)[0]

    def run_saved(self, x, residual=None, out=None):
        """-> (y, saved): the pre-activations that `backward` needs, fp32 [rows, out]; None without an activation."""
        return self._forward(x, residual, out, True)

    def backward(self, dy, x, saved, need=("x", "weight", "bias")):
        """Gradients for dy, the gradient of y: -> (dx, dweight, dbias), None for what `need` leaves out or the layer lacks.
        x and saved are those of the forward call.  The gradient of its residual is dy."""
        x2, xs = self._rows(x, self.in_features, "x")
        rows = x2.shape[0]
        _need(tuple(dy.shape) == tuple(x.shape[:-1]) + (self.out_features,), "dy: the shape of y expected")
        d2, ds = self._rows(dy, self.out_features, "dy", rows)
        if self.act != "none":
            self._saved(saved, (rows, self.out_features))
        new = lambda shape, t: torch.empty(shape, dtype=t, device=self.device)  # noqa: E731
        dx = new(tuple(x.shape), self.dtype) if "x" in need else None
        dw = new((self.out_features, self.in_features), self.dtype) if "weight" in need else None
        db = new((self.out_features,), torch.float32) if "bias" in need and self.bias is not None else None
        self._call("dlf_linear_backward", rows, (xs, 0, 0, ds), d2, x2, self.weight, saved if self.act != "none" else None, dx, dw, db)
        return dx, dw, db


class GatedLinear(_Operator):
    """h = act(x w_gate^T + b_gate) * (x w_up^T + b_up).  w_gate, w_up [out, in], of one type and row distance (two halves of one
    tensor among others), biases fp32 [out] or None."""

    def __init__(self, w_gate, w_up, b_gate=None, b_up=None, act="silu"):
        self.w_gate, self.w_up = _weight(w_gate, "w_gate"), _weight(w_up, "w_up")
        _need(w_up.shape == w_gate.shape and w_up.dtype == w_gate.dtype and w_up.device == w_gate.device and
              _stride(w_up, "w_up") == _stride(w_gate, "w_gate"), "w_up: shape, type, device and row distance of w_gate expected")
        self._setup(w_gate, act)
        self.b_gate, self.b_up = (_bias(b, self.out_features, w_gate, n) for b, n in ((b_gate, "b_gate"), (b_up, "b_up")))

    def _forward(self, x, out, save):
        x2, xs = self._rows(x, self.in_features, "x")
        rows = x2.shape[0]
        out, o2, ys = self._out(out, x.shape[:-1] + (self.out_features,), rows)
        saved = torch.empty((2, rows, self.out_features), dtype=torch.float32, device=self.device) if save else None
        self._call("dlf_gated", rows, (xs, ys, 0, 0), x2, self.w_gate, self.w_up, self.b_gate, self.b_up, o2, saved)
        return out, saved

    def run(self, x, out=None):
        """-> h [..., out]; written to `out` if given."""
        return self._forward(x, out, False)[0]

    def run_saved(self, x, out=None):
        """-> (h, saved): both projections' results, which `backward` needs, fp32 [2, rows, out]."""
        return self._forward(x, out, True)

    def backward(self, dh, x, saved, need=("x", "weight", "bias")):
        """Gradients for dh, the gradient of h: -> (dx, dw_gate, dw_up, db_gate, db_up), None for what `need` leaves out or the
        layer lacks.  x and saved are those of the forward call."""
        x2, xs = self._rows(x, self.in_features, "x")
        rows = x2.shape[0]
        _need(tuple(dh.shape) == tuple(x.shape[:-1]) + (self.out_features,), "dh: the shape of h expected")
        d2, ds = self._rows(dh, self.out_features, "dh", rows)
        self._saved(saved, (2, rows, self.out_features))
        new = lambda shape, t: torch.empty(shape, dtype=t, device=self.device)  # noqa: E731
        dx = new(tuple(x.shape), self.dtype) if "x" in need else None
        dw = [new((self.out_features, self.in_features), self.dtype) if "weight" in need else None for _ in range(2)]
        db = [new((self.out_features,), torch.float32) if "bias" in need and b is not None else None for b in (self.b_gate, self.b_up)]
        self._call("dlf_gated_backward", rows, (xs, 0, 0, ds), d2, x2, self.w_gate, self.w_up, saved, dx, *dw, *db)
        return (dx, *dw, *db)


class FeedForward:
    """The block y = down(gated(x)) + residual: two kernels forward."""

    def __init__(self, gated, down):
        _need(isinstance(gated, GatedLinear) and isinstance(down, Linear), "a GatedLinear and a Linear expected")
        _need(down.in_features == gated.out_features and down.dtype == gated.dtype and down.device == gated.device,
              "down: %d input features of type %s on %s expected", gated.out_features, gated.dtype, gated.device)
        self.gated, self.down = gated, down

    def run(self, x, residual=None, out=None):
        """-> y [..., out]; `out` may be x itself where x is the residual."""
        return self.down.run(self.gated.run(x), residual, out)

    def run_saved(self, x, residual=None, out=None):
        """-> (y, saved): what `backward` needs."""
        h, saved_g = self.gated.run_saved(x)
        y, saved_d = self.down.run_saved(h, residual, out)
        return y, (h, saved_g, saved_d)

    def backward(self, dy, x, saved, need=("x", "weight", "bias")):
        """-> (dx, (dw_gate, dw_up, db_gate, db_up), (dw_down, db_down)).  dx is the gradient through the products; where x
        was the residual too, dy is added to it by the caller."""
        h, saved_g, saved_d = saved
        dh, dw, db = self.down.backward(dy, h, saved_d, tuple(set(need) | {"x"}))
        g = self.gated.backward(dh, x, saved_g, need)
        return g[0], g[1:], (dw, db)
