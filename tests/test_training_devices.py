"""Every tensor of a call of the root-mean-square norm, a head's cross entropy and distillation has to be on the GPU that
the call runs on and have the shape and type that it says.  Checked without a GPU, on tensors that say where they are;
the library is not reached."""
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


N, D, V, K = 4, 16, 64, 5
f32, i64, i32 = torch.float32, torch.int64, torch.int32
CALLS = {
    "rms_norm": {"x": (N, D), "weight": (D,), "residual": (N, D), "out": (N, D), "h": (N, D)},
    "rms_norm_fp8": {"x": (N, D), "weight": (D,), "residual": (N, D), "h": (N, D)},
    "rms_norm_backward": {"dy": (N, D), "h": (N, D), "rstd": (N,), "weight": (D,), "dh": (N, D), "out": (N, D)},
    "linear_cross_entropy": {"X": (N, D), "W": (V, D), "targets": (N,)},
    "linear_cross_entropy_backward": {"dloss": (N,), "X": (N, D), "W": (V, D), "targets": (N,), "stats": (N, 2)},
    "distillation_loss": {"logits": (N, V), "top_idx": (N, K), "top_logp": (N, K)},
    "distillation_loss_backward": {"dloss": (N,), "logits": (N, V), "top_idx": (N, K), "top_logp": (N, K), "stats": (N, 4), "out": (N, V)},
}
TYPES = {"targets": i64, "top_idx": i32}
STATUS = ("linear_cross_entropy", "linear_cross_entropy_backward", "distillation_loss")
WORKSPACE = ("rms_norm_backward", "linear_cross_entropy", "linear_cross_entropy_backward", "distillation_loss")


def names(call):
    return [*CALLS[call], *(["status"] if call in STATUS else []), *(["workspace"] if call in WORKSPACE else [])]


def arguments(call, bad=None, at=0):
    args = {name: Placed.on(torch.zeros(shape, dtype=TYPES.get(name, f32)), at if name == bad else 0) for name, shape in CALLS[call].items()}
    if call in STATUS:
        args["status"] = Placed.on(torch.zeros(1, dtype=i32), at if bad == "status" else 0)
    if call in WORKSPACE:
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


ALL = [(c, n) for c in CALLS for n in names(c)]


@pytest.mark.parametrize("call", list(CALLS))
def test_in_place_all_reach_the_library(call):
    with pytest.raises(Reached):
        getattr(cci, call)(**arguments(call))


@pytest.mark.parametrize("at", [HOST, 1])
@pytest.mark.parametrize("call,name", ALL)
def test_a_tensor_elsewhere_is_refused(call, name, at):
    with pytest.raises(ValueError):
        getattr(cci, call)(**arguments(call, name, at))


@pytest.mark.parametrize("call", list(CALLS))
def test_all_on_another_than_the_current_gpu_are_refused(call):
    with pytest.raises(ValueError):
        getattr(cci, call)(**{k: Placed.on(t, 1) for k, t in arguments(call).items()})


@pytest.mark.parametrize("call,name", [(c, n) for c, n in ALL if n not in ("status", "workspace")])
def test_another_shape_is_refused(call, name):
    args = arguments(call)
    t = args[name]
    shape = list(t.shape)
    first = {"x", "X", "logits", "h", "W"}  # what the call takes its sizes from
    if name in first and (name != "h" or call == "rms_norm_backward"):
        shape = [*shape, 1]
    else:
        shape[0] += 1
    args[name] = Placed.on(torch.zeros(shape, dtype=t.dtype), 0)
    with pytest.raises((ValueError, RuntimeError)):
        getattr(cci, call)(**args)


@pytest.mark.parametrize("call,name", [(c, n) for c, n in ALL if n not in ("workspace",)])
def test_another_type_is_refused(call, name):
    args = arguments(call)
    args[name] = Placed.on(args[name].to(torch.float64), 0)
    with pytest.raises((ValueError, TypeError)):
        getattr(cci, call)(**args)


@pytest.mark.parametrize("call,name", [(c, n) for c, n in ALL if n not in ("status",)])
def test_elements_apart_are_refused(call, name):
    args = arguments(call)
    t = args[name]
    wide = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype)
    args[name] = Placed.on(wide[..., ::2], 0)
    with pytest.raises(ValueError):
        getattr(cci, call)(**args)


@pytest.mark.parametrize("call", ["rms_norm", "rms_norm_fp8"])
def test_h_without_a_residual_is_refused(call):
    args = arguments(call)
    del args["residual"]
    with pytest.raises(ValueError):
        getattr(cci, call)(**args)


def test_rows_with_strides_are_taken():
    wide = Placed.on(torch.zeros((N, 3 * D)), 0)
    args = arguments("rms_norm")
    args["x"] = Placed.on(wide[:, 3:3 + D], 0)
    with pytest.raises(Reached):
        cci.rms_norm(**args)
