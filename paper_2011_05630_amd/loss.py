"""The softmax cross entropy of a linear layer over many classes (a vocabulary), without its logits in memory, and its gradients, which keep two bytes
for each logit of a piece of the rows.

The object holds the caller's weight and bias, as the feed-forward operators do, and takes the same tensors: fp16 or bf16, of one type, rows of
consecutive elements at any alignment and any distance below 2^24 elements, biases and their gradients fp32, any number of leading dimensions; targets int64.  Every call runs on
the current stream of the weight's device, asynchronously; outputs and workspaces come from PyTorch's allocator, so calls may be captured into
a graph.  Automatic differentiation does not see the calls: call under torch.no_grad(), or inside a torch.autograd.Function's forward
and backward.
"""
from .feedforward import _GRADIENTS, _bias, _native, _need, _Operator, _stream, _stride, _wanted, _weight


class CrossEntropy(_Operator):
    """loss[r] = log sum_c exp(z[r][c]) - z[r][target[r]], z = x weight^T + bias.  weight [classes, in], bias fp32 [classes] or None (a class
    whose bias is -inf takes no part).  A row whose target is `ignore_index` has loss 0 and no gradient; any other target that is no class gives NaN.

    piece_bytes: what dz of a piece of the rows may take, two bytes a class (256 rows at least).  `gradients` with the bias's among them keeps the piece's
    logits beside it, twice that much: up to three times piece_bytes in all."""

    def __init__(self, weight, bias=None, ignore_index=-100, piece_bytes=1 << 30):
        self.weight = _weight(weight, "weight")
        self.bias = _bias(bias, weight.shape[0], weight, "bias")
        _need(isinstance(ignore_index, int) and -(1 << 63) <= ignore_index < 1 << 63, "ignore_index: a whole number of 64 bits expected")
        _need(isinstance(piece_bytes, int) and 0 < piece_bytes < 1 << 50, "piece_bytes: a number above 0 expected")
        self.dtype, self.device, self.ignore_index, self.piece_bytes = weight.dtype, weight.device, ignore_index, piece_bytes
        self.classes, self.in_features = weight.shape
        self._index = weight.get_device()
        op = _native().CrossEntropy(weight, bias, _stride(weight, "weight"), ignore_index, piece_bytes)
        self._forward, self._backward, self._gradients = op.forward, op.backward, op.gradients
        self._fixed = frozenset(self.__dict__)

    def run(self, x, target):
        """-> loss, fp32, of the leading dimensions of x."""
        return self._forward(x, target, False, _stream(self._index))

    def run_saved(self, x, target):
        """-> (loss, lse): lse, the logarithm of the sum of exponentials, is what `backward` needs."""
        return self._forward(x, target, True, _stream(self._index))

    def backward(self, dloss, x, target, lse, dlse=None, need=_GRADIENTS):
        """Gradients for dloss and dlse, the gradients of loss and lse: fp32 tensors of their shape or of one element (the same for every row), dloss
        also a number: -> (dx, dweight, dbias), None for what `need` leaves out or the layer lacks.  x, target and lse are those of the forward
        call.  lse in 32 bits leaves every probability off by up to 2^-24 |lse| of itself, which `gradients` does not; and the logits that it was formed
        of may come from other kernels than those of this call, with their sums in another order."""
        return self._backward(dloss, x, target, lse, dlse, *_wanted(need), _stream(self._index))

    def gradients(self, x, target, dloss, need=_GRADIENTS):
        """-> (loss, dx, dweight, dbias): run and backward in one, for a dloss that is known beforehand: a mean's 1 / rows, a loss scale.  It takes a quarter less."""
        return self._gradients(x, target, dloss, *_wanted(need), _stream(self._index))
