"""Which tensors the general path of the 4-bit operators refuses before it calls the library: those whose memory a kernel cannot reach, and those of another shape.  No
GPU: `OnGpu` tensors say that they lie on one, and the library is replaced by one that writes down its calls."""
import ctypes
import types

import pytest
import torch

from paper_2603_05232_amd import binding

M, K, O, E, TOP = 6, 300, 40, 3, 2
U8, I32, F32, BF16 = torch.uint8, torch.int32, torch.float32, torch.bfloat16


class OnGpu(torch.Tensor):
    """A tensor on the first GPU, as far as a caller can ask."""
    is_cuda = True

    def get_device(self):
        return 0


class OnAnotherGpu(OnGpu):
    def get_device(self):
        return 1


def there(shape, dtype):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """The library's sizes, and its launches as a list."""

    def __init__(self, real):
        self.real, self.launched = real, []

    def __getattr__(self, name):
        if name in ("mx4_row_bytes", "mx4_row_scales", "mx4_packed_sizes", "mx4_gemm_workspace_bytes", "expert_route_workspace_bytes"):
            return getattr(self.real, name)

        def launch(*args):
            self.launched.append(name)
            return 0
        return launch


@pytest.fixture
def library(monkeypatch):
    lib = Library(binding.load())
    names = ("mx4_quant", "mx4_dequant", "mx4_product", "expert_route", "expert_combine")
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(binding, "_mx4_calls", types.SimpleNamespace(**dict.fromkeys(names, lambda *args: None)))
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    return lib


def operands():
    """Every operator's tensors by name, and the call that takes them."""
    wv, wm = binding.mx4_packed_sizes(O, K)
    ev, em = binding.mx4_packed_sizes(O, K, experts=E)
    code = lambda: there((M, 256), U8)  # noqa: E731
    scale = lambda: there((2, M, 8), U8)  # noqa: E731
    ws = lambda: there((4096,), U8)  # noqa: E731
    return {
        "mx4_quant": (dict(X=there((M, K), BF16), rows=there((M,), I32), codes=code(), scales=scale()), lambda t: binding.mx4_quant(t["X"], t["rows"], t["codes"], t["scales"])),
        "mx4_dequant": (dict(codes=code(), scales=scale(), out=there((M, K), F32)), lambda t: binding.mx4_dequant(t["codes"], t["scales"], K, out=t["out"])),
        "mx4_pack": (dict(codes=code(), scales=scale()), lambda t: binding.mx4_pack(t["codes"], t["scales"], K)),
        "mx4_gemm": (dict(codes=code(), scales=scale(), w_vals=there((wv,), U8), w_meta=there((wm,), U8), out=there((M, O), BF16), workspace=ws()),
                     lambda t: binding.mx4_gemm(t["codes"], t["scales"], t["w_vals"], t["w_meta"], O, K, out=t["out"], workspace=t["workspace"])),
        "mx4_grouped_gemm": (dict(codes=code(), scales=scale(), offsets=there((E + 1,), I32), w_vals=there((ev,), U8), w_meta=there((em,), U8), out=there((M, O), BF16), workspace=ws()),
                             lambda t: binding.mx4_grouped_gemm(t["codes"], t["scales"], t["offsets"], t["w_vals"], t["w_meta"], O, K, out=t["out"], workspace=t["workspace"])),
        "expert_route": (dict(logits=there((M, E), F32), workspace=ws()), lambda t: binding.expert_route(t["logits"], TOP, workspace=t["workspace"])),
        "expert_combine": (dict(Y=there((M * TOP, O), BF16), slots=there((M, TOP), I32), weights=there((M, TOP), F32), base=there((M, O), BF16), out=there((M, O), BF16)),
                           lambda t: binding.expert_combine(t["Y"], t["slots"], t["weights"], base=t["base"], out=t["out"])),
    }


NAMES = {"mx4_quant": ("X", "rows", "codes", "scales"), "mx4_dequant": ("codes", "scales", "out"), "mx4_pack": ("codes", "scales"),
         "mx4_gemm": ("codes", "scales", "w_vals", "w_meta", "out", "workspace"), "mx4_grouped_gemm": ("codes", "scales", "offsets", "w_vals", "w_meta", "out", "workspace"),
         "expert_route": ("logits", "workspace"), "expert_combine": ("Y", "slots", "weights", "base", "out")}
EACH = [(op, name) for op, names in NAMES.items() for name in names]


@pytest.mark.parametrize("op", NAMES)
def test_tensors_on_the_gpu_are_taken(library, op):
    tensors, call = operands()[op]
    assert set(tensors) == set(NAMES[op])
    call(tensors)
    assert library.launched == [op]


@pytest.mark.parametrize("op,name", EACH)
def test_a_tensor_in_host_memory_is_refused(library, op, name):
    tensors, call = operands()[op]
    tensors[name] = torch.zeros(tensors[name].shape, dtype=tensors[name].dtype)
    with pytest.raises(AssertionError):
        call(tensors)
    assert library.launched == []


@pytest.mark.parametrize("op,name", [e for e in EACH if e[1] != NAMES[e[0]][0]])
def test_a_tensor_on_another_gpu_than_the_first_is_refused(library, op, name):
    tensors, call = operands()[op]
    tensors[name] = tensors[name].as_subclass(torch.Tensor).as_subclass(OnAnotherGpu)
    with pytest.raises(AssertionError):
        call(tensors)
    assert library.launched == []


@pytest.mark.parametrize("op", ["mx4_gemm", "mx4_grouped_gemm", "expert_route"])
def test_a_workspace_in_pieces_is_refused(library, op):
    tensors, call = operands()[op]
    tensors["workspace"] = there((1,), U8).expand(4096)         # one byte that says it is 4096
    with pytest.raises(AssertionError):
        call(tensors)
    assert library.launched == []


@pytest.mark.parametrize("op,name", [("mx4_gemm", "w_vals"), ("mx4_gemm", "w_meta"), ("mx4_grouped_gemm", "w_vals"), ("mx4_grouped_gemm", "w_meta")])
def test_packed_weights_of_another_type_are_refused(library, op, name):
    tensors, call = operands()[op]
    tensors[name] = tensors[name].view(torch.int8)
    with pytest.raises(AssertionError):
        call(tensors)
    assert library.launched == []


@pytest.mark.parametrize("op,name", [("mx4_quant", "rows"), ("mx4_grouped_gemm", "offsets")])
def test_lists_of_two_dimensions_are_refused(library, op, name):
    """Their first dimension alone would be taken for the number of rows, or of experts."""
    tensors, call = operands()[op]
    tensors[name] = there((tensors[name].numel(), 2), I32)
    with pytest.raises(AssertionError):
        call(tensors)
    assert library.launched == []
