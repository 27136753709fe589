"""Every tensor of a call of the layers around a pruned projection has to be on the GPU that the call runs on: an
address of the host or of another GPU must not reach a kernel.  Checked without a GPU, on tensors that say where they
are; the library is not reached."""
import pytest
import torch

import paper_1910_11971_gb300 as cci

HOST = -1


class Placed(torch.Tensor):
    """A host tensor that says it is on GPU `at`."""

    @staticmethod
    def on(t, at):
        r = torch.Tensor._make_subclass(Placed, t)
        r.at = at
        return r

    def get_device(self):
        return self.at

    @property
    def is_cuda(self):
        return self.at >= 0


N, D, F, V, G, K = 4, 16, 32, 64, 8, 2
f32 = torch.float32
NORM = {"x": (N, D), "weight": (D,), "bias": (D,), "out": (N, D)}
NORM_BACKWARD = {"dy": (N, D), "x": (N, D), "mean": (N,), "rstd": (N,), "weight": (D,), "out": (N, D)}
LOGPROBS = {"logits": (N, V), "tokens": (N,)}
LOGPROBS_BACKWARD = {"logits": (N, V), "tokens": (N,), "stats": (N, 2), "dlogp": (N,), "entropy": (N,), "dentropy": (N,), "out": (N, V)}
GATED = {"X": (N, D), "Wg": (F, D), "Wu": (F, D), "out": (N, F)}
GATED_BACKWARD = {"dH": (N, F), "X": (N, D), "Wg": (F, D), "Wu": (F, D), "g": (N, F), "u": (N, F)}
CALLS = {"layer_norm": NORM, "layer_norm_backward": NORM_BACKWARD, "token_logprobs": LOGPROBS,
         "token_logprobs_backward": LOGPROBS_BACKWARD, "gated_linear": GATED, "gated_linear_backward": GATED_BACKWARD}
WITH_WORKSPACE = ("layer_norm_backward", "gated_linear", "gated_linear_backward", "gated_linear_packed")


def arguments(call, bad=None, at=0):
    args = {}
    for name, shape in CALLS[call].items():
        t = torch.zeros(shape, dtype=torch.int64 if name == "tokens" else f32)
        args[name] = Placed.on(t, at if name == bad else 0)
    if call != "layer_norm":
        args["status"] = Placed.on(torch.zeros(1, dtype=torch.int32), at if bad == "status" else 0)
    if call in WITH_WORKSPACE:
        args["workspace"] = Placed.on(torch.zeros(1 << 16, dtype=torch.uint8), at if bad == "workspace" else 0)
    return args


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    class Library:
        def __getattr__(self, name):
            def reached(*args):
                raise Reached
            return reached

    monkeypatch.setattr(cci, "lib", Library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


@pytest.mark.parametrize("at", [HOST, 1])
@pytest.mark.parametrize("call,name", [(c, n) for c, names in CALLS.items() for n in
                                       [*names, *(["status"] if c != "layer_norm" else []), *(["workspace"] if c in WITH_WORKSPACE else [])]])
def test_a_tensor_elsewhere_is_refused(call, name, at):
    with pytest.raises(ValueError):
        getattr(cci, call)(**arguments(call, name, at))


@pytest.mark.parametrize("at", [HOST, 1])
@pytest.mark.parametrize("place", range(5))
def test_packed_weights_elsewhere_are_refused(place, at):
    where = [at if place == i else 0 for i in range(5)]
    v, i = torch.zeros((F // G, D, K)), torch.zeros((F // G, D, K), dtype=torch.uint8)
    with pytest.raises(ValueError):
        cci.gated_linear_packed(Placed.on(torch.zeros((N, D)), where[0]), (Placed.on(v, where[1]), Placed.on(i, where[2])),
                                (Placed.on(v, where[3]), Placed.on(i, where[4])), F, G, K,
                                workspace=Placed.on(torch.zeros(1 << 16, dtype=torch.uint8), 0))


@pytest.mark.parametrize("call", list(CALLS))
def test_all_on_another_than_the_current_gpu_are_refused(call):
    args = {k: Placed.on(t, 1) for k, t in arguments(call).items()}
    with pytest.raises(ValueError):
        getattr(cci, call)(**args)


@pytest.mark.parametrize("call", list(CALLS))
def test_in_place_all_reach_the_library(call):
    with pytest.raises(Reached):
        getattr(cci, call)(**arguments(call))


@pytest.mark.parametrize("status", [torch.zeros(1), torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)])
def test_a_status_word_is_a_32_bit_integer(status):
    args = arguments("layer_norm_backward")
    args["status"] = Placed.on(status, 0)
    with pytest.raises(ValueError):
        cci.layer_norm_backward(**args)


def test_the_workspace_is_one_piece():
    args = arguments("gated_linear")
    args["workspace"] = Placed.on(torch.zeros(1 << 16, dtype=torch.uint8)[::2], 0)
    with pytest.raises(ValueError):
        cci.gated_linear(**args)
