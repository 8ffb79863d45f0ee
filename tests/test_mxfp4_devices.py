"""CPU-only checks of where the operands of the layer norm and MXFP4 calls may be: in the memory of one GPU, which
is the current device while the call is made.  Tensors say that they are on a GPU, the library's calls are written down, and nothing is
launched."""
import contextlib

import pytest
import torch

import paper_2410_20046_amd as dq
from paper_2410_20046_amd import binding


class Claims(torch.Tensor):
    """A tensor in host memory that says it is on GPU `gpu`."""

    gpu = 0
    is_cuda = True

    def get_device(self):
        return self.gpu


def on(gpu, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Claims)
    t.gpu = gpu
    return t


def space(gpu):
    return on(gpu, 1 << 16, dtype=torch.uint8)


def matrix(gpu, rows, cols):
    groups = -(-cols // 128)
    make = lambda n: on(gpu, rows, n, dtype=torch.uint8) if gpu >= 0 else torch.zeros(rows, n, dtype=torch.uint8)  # noqa: E731
    return dq.MxMatrix(rows, cols, codes=make(64 * groups), scales=make(4 * groups))


class Library:
    """The library's entry points; each writes down its name, its stream and the device that is current."""

    def __init__(self):
        self.calls, self.current = [], 0

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args[-1], self.current)) or 0


@pytest.fixture
def library(monkeypatch):
    made = Library()

    @contextlib.contextmanager
    def device(gpu):
        before, made.current = made.current, gpu
        yield
        made.current = before

    monkeypatch.setattr(binding, "lib", lambda: made)
    monkeypatch.setattr(binding, "_raw_stream", lambda gpu: 0 if gpu == 0 else 100 + gpu)
    monkeypatch.setattr(binding, "_current_device", lambda: made.current, raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    return made


M, N, K = 4, 6, 64


def operands(call):
    """name -> how to make it on a GPU, of each of a call's operands; the first one says which GPU it is."""
    put = lambda *shape: lambda gpu: on(gpu, *shape) if gpu >= 0 else torch.zeros(*shape)  # noqa: E731
    ws = lambda gpu: space(gpu) if gpu >= 0 else torch.zeros(1 << 16, dtype=torch.uint8)  # noqa: E731
    held = lambda *shape: lambda gpu: matrix(gpu, *shape)  # noqa: E731
    return {
        "quant": dict(x=put(M, K), by_rows=held(M, K), by_cols=held(K, M), gate=put(M, K), col_sums=put(K), workspace=ws),
        "dequant": dict(out=put(M, K), q=held(M, K)),
        "matmul": dict(out=put(M, N), a=held(M, K), b=held(N, K), bias=put(N), workspace=ws),
        "linear": dict(x=put(M, K), w=held(N, K), out=put(M, N), bias=put(N), gamma=put(K), beta=put(K), workspace=ws),
        "norm": dict(x=put(M, K), gamma=put(K), beta=put(K), y=put(M, K), mean=put(M), rstd=put(M), q=held(M, K)),
        "norm_bwd": dict(x=put(M, K), dy=put(M, K), mean=put(M), rstd=put(M), gamma=put(K), dx=put(M, K), dgamma=put(K), dbeta=put(K), workspace=ws),
    }[call]


CALLS = {"quant": dq.dqrm_mxfp4_quant, "dequant": dq.dqrm_mxfp4_dequant, "matmul": dq.dqrm_mxfp4_matmul, "linear": dq.dqrm_mxfp4_linear,
         "norm": dq.dqrm_layernorm_fwd, "norm_bwd": dq.dqrm_layernorm_bwd}


def make(call, gpus, **others):
    args = {name: f(gpus.get(name, gpus["all"])) for name, f in operands(call).items()}
    if call in ("norm", "linear"):
        args["eps"] = 1e-5
    CALLS[call](**args, **others)


@pytest.mark.parametrize("call", CALLS)
def test_an_operand_in_host_memory_is_refused(call, library):
    for name in operands(call):
        with pytest.raises(dq.DqrmError) as e:
            make(call, {"all": 0, name: -1})
        assert e.value.code == dq.ERR_INVALID_ARG, name
    with pytest.raises(dq.DqrmError) as e:
        make(call, {"all": -1})
    assert e.value.code == dq.ERR_INVALID_ARG
    with pytest.raises(dq.DqrmError):
        make(call, {"all": -1}, stream=0)
    assert not library.calls


@pytest.mark.parametrize("call", CALLS)
def test_an_operand_on_another_gpu_is_refused(call, library):
    for name in operands(call):
        with pytest.raises(dq.DqrmError) as e:
            make(call, {"all": 0, name: 1})
        assert e.value.code == dq.ERR_INVALID_ARG, name
    assert not library.calls


def test_a_matrix_is_not_in_parts_on_two_devices():
    with pytest.raises(dq.DqrmError):
        dq.MxMatrix(4, 64, codes=on(0, 4, 64, dtype=torch.uint8), scales=torch.zeros(4, 4, dtype=torch.uint8))


def test_rows_on_top_of_each_other_are_left_to_the_library(monkeypatch):
    """The library's own refusal, before anything is launched."""
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    with pytest.raises(dq.DqrmError) as e:
        dq.dqrm_mxfp4_quant(on(0, 1, 64).expand(4, 64), matrix(0, 4, 64), stream=0)
    assert e.value.code == dq.ERR_INVALID_ARG and "operands" not in str(e.value)


@pytest.mark.parametrize("call", CALLS)
def test_a_call_is_made_on_the_gpu_that_holds_its_operands(call, library):
    for current in (0, 1):
        for gpu in (0, 1, 3):
            library.current, library.calls = current, []
            make(call, {"all": gpu})
            make(call, {"all": gpu}, stream=77)
            assert [c[1:] for c in library.calls] == [(0 if gpu == 0 else 100 + gpu, gpu), (77, gpu)]
            assert library.current == current


def test_a_matrix_is_made_where_its_calls_need_it(monkeypatch):
    """On the current GPU if there is one and the default device is the host; beside the codes that are given."""
    made = []
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: made.append(device) or real(*a, **k))
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    dq.MxMatrix(4, 64)
    assert [torch.device(d).type for d in made] == ["cuda", "cuda"]
    made.clear()
    dq.MxMatrix(4, 64, codes=torch.zeros(4, 64, dtype=torch.uint8))
    assert [torch.device(d).type for d in made] == ["cpu"]
    made.clear()
    monkeypatch.setattr(torch, "get_default_device", lambda: torch.device("cuda:1"))
    dq.MxMatrix(4, 64)
    assert [torch.device(d) for d in made] == [torch.device("cuda:1")] * 2
