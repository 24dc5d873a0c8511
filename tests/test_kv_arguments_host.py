"""Which tensors the general path of the cache's operators refuses before it calls the library: those whose memory a kernel cannot reach, those on another GPU than the
current one, and those of another shape or type.  No GPU, as in test_mx4_arguments_host."""
import types

import pytest
import torch

from paper_2603_05232_amd import binding
from test_mx4_arguments_host import BF16, F32, I32, U8, OnAnotherGpu, there

B, W, N, Hq, H, D, PAGE, P = 3, 4, 10, 4, 2, 40, 32, 7
SIZES = ("kv_page_bytes", "kv_tables_workspace_bytes", "kv_attention_workspace_bytes")


class Library:
    def __init__(self, real):
        self.real, self.launched = real, []

    def __getattr__(self, name):
        if name in SIZES:
            return getattr(self.real, name)

        def launch(*args):
            self.launched.append(name)
            return 0
        return launch


@pytest.fixture
def library(monkeypatch):
    lib = Library(binding.load())
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(binding, "_kv_calls", types.SimpleNamespace(**dict.fromkeys(("kv_tables", "kv_write", "kv_read", "kv_attention"), lambda *args: None)))
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    return lib


def operands():
    """Every operator's tensors by name, and the call that takes them."""
    pages = lambda: there((P, binding.kv_page_bytes(H, PAGE, D, "i8")), U8)  # noqa: E731
    rows = lambda: there((N, H, D), BF16)  # noqa: E731
    return {
        "kv_tables": (dict(lens=there((B,), I32), want=there((B,), I32), table=there((B, W), I32), pool=there((P,), I32), left=there((1,), I32), new_lens=there((B,), I32),
                           new_left=there((1,), I32), workspace=there((1 << 16,), U8)),
                      lambda t: binding.kv_tables(t["lens"], t["want"], t["table"], t["pool"], t["left"], PAGE, N, t["new_lens"], t["new_left"], t["workspace"])),
        "kv_write": (dict(K=rows(), V=rows(), slots=there((N,), I32), pages=pages()), lambda t: binding.kv_write(t["K"], t["V"], t["slots"], t["pages"], PAGE, "i8")),
        "kv_read": (dict(pages=pages(), slots=there((N,), I32), K=rows(), V=rows()), lambda t: binding.kv_read(t["pages"], t["slots"], H, D, PAGE, "i8", K=t["K"], V=t["V"])),
        "kv_attention": (dict(q=there((B, Hq, D), F32), pages=pages(), table=there((B, W), I32), lens=there((B,), I32), out=there((B, Hq, D), BF16), workspace=there((4096,), U8)),
                         lambda t: binding.kv_attention(t["q"], t["pages"], t["table"], t["lens"], H, PAGE, "i8", out=t["out"], workspace=t["workspace"])),
    }


NAMES = {op: tuple(tensors) for op, (tensors, _) in {
    "kv_tables": (("lens", "want", "table", "pool", "left", "new_lens", "new_left", "workspace"), 0), "kv_write": (("K", "V", "slots", "pages"), 0),
    "kv_read": (("pages", "slots", "K", "V"), 0), "kv_attention": (("q", "pages", "table", "lens", "out", "workspace"), 0)}.items()}
EACH = [(op, name) for op, names in NAMES.items() for name in names]


def refused(library, op, tensors, errors=AssertionError):
    with pytest.raises(errors):
        operands()[op][1](tensors)
    assert library.launched == []


@pytest.mark.parametrize("op", NAMES)
def test_tensors_on_the_gpu_are_taken(library, op):
    tensors, call = operands()[op]
    assert tuple(tensors) == NAMES[op]
    call(tensors)
    assert library.launched == [op]


@pytest.mark.parametrize("op,name", EACH)
def test_a_tensor_in_host_memory_is_refused(library, op, name):
    tensors = operands()[op][0]
    tensors[name] = torch.zeros(tensors[name].shape, dtype=tensors[name].dtype)
    refused(library, op, tensors)


@pytest.mark.parametrize("op,name", EACH)
def test_a_tensor_on_another_gpu_is_refused(library, op, name):
    tensors = operands()[op][0]
    tensors[name] = tensors[name].as_subclass(torch.Tensor).as_subclass(OnAnotherGpu)
    refused(library, op, tensors)


@pytest.mark.parametrize("op", NAMES)
def test_tensors_on_another_gpu_than_the_current_one_are_refused(library, monkeypatch, op):
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    refused(library, op, operands()[op][0])


@pytest.mark.parametrize("op,name", [(op, n) for op, n in EACH if n in ("lens", "want", "table", "pool", "left", "slots", "new_lens", "new_left")])
def test_numbers_of_another_type_are_refused(library, op, name):
    tensors = operands()[op][0]
    tensors[name] = there(tensors[name].shape, torch.int64)
    refused(library, op, tensors, TypeError)


@pytest.mark.parametrize("op,name", EACH)
def test_another_number_of_dimensions_is_refused(library, op, name):
    tensors = operands()[op][0]
    if name == "workspace":
        pytest.skip("any shape will do")
    tensors[name] = there((*tensors[name].shape, 1), tensors[name].dtype)
    refused(library, op, tensors, (AssertionError, ValueError))


@pytest.mark.parametrize("op,name", [(op, n) for op, n in EACH if n not in ("workspace", "pool", "table", "pages")])
def test_one_row_less_is_refused(library, op, name):
    tensors = operands()[op][0]
    tensors[name] = there((tensors[name].shape[0] - 1, *tensors[name].shape[1:]), tensors[name].dtype)
    refused(library, op, tensors)


@pytest.mark.parametrize("op,name,dtype", [("kv_write", "pages", torch.int8), ("kv_read", "pages", torch.int8), ("kv_attention", "pages", torch.int8), ("kv_attention", "out", F32), ("kv_write", "V", F32),
                                           ("kv_read", "V", F32)])
def test_another_type_is_refused(library, op, name, dtype):
    tensors = operands()[op][0]
    tensors[name] = there(tensors[name].shape, dtype)
    refused(library, op, tensors)


@pytest.mark.parametrize("op,name", [("kv_write", "K"), ("kv_write", "V"), ("kv_read", "K"), ("kv_read", "V"), ("kv_attention", "q"), ("kv_attention", "out")])
def test_heads_in_pieces_are_refused(library, op, name):
    tensors = operands()[op][0]
    t = tensors[name]
    tensors[name] = there((*t.shape[:2], 2 * D), t.dtype)[:, :, ::2]
    refused(library, op, tensors)


@pytest.mark.parametrize("op", ["kv_tables", "kv_attention"])
def test_a_workspace_in_pieces_is_refused(library, op):
    tensors = operands()[op][0]
    tensors["workspace"] = there((1,), U8).expand(1 << 16)
    refused(library, op, tensors)
