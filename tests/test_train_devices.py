"""CPU-only checks of where the operands of the residual norms, the loss and the clip may be: in the memory of one GPU, which is the current
device while the call is made.  Tensors say that they are on a GPU, the library's calls are written down, and nothing is launched."""
import pytest
import torch

import paper_2410_20046_amd as dq
from test_mxfp4_devices import library, matrix, on, space  # noqa: F401  (library: the fixture)

M, V, K = 4, 6, 64


def put(*shape, dtype=torch.float32):
    return lambda gpu: on(gpu, *shape, dtype=dtype) if gpu >= 0 else torch.zeros(*shape, dtype=dtype)


def room(gpu):
    return space(gpu) if gpu >= 0 else torch.zeros(1 << 16, dtype=torch.uint8)


def block(gpu):
    return dq.ResidualNorm(post=dq.NORM_RMS, post_gamma=put(K)(gpu), gate=put(K)(gpu))


def tensors(gpu):
    return dq.Grads([put(M, K)(gpu), put(7)(gpu)], out=[put(M, K)(gpu), put(7)(gpu)], counts={0: put(1, dtype=torch.int32)(gpu)})


# name -> how to make it on a GPU, of each of a call's operands
OPERANDS = {
    "norm": (dq.dqrm_residual_norm_fwd, dict(u=put(M, K), norm=block, r=put(M, K), out=put(M, K), y=put(M, K), stats=put(4, M), q=lambda gpu: matrix(gpu, M, K))),
    "norm_bwd": (dq.dqrm_residual_norm_bwd, dict(dout=put(M, K), norm=block, dy=put(M, K), u=put(M, K), out=put(M, K), stats=put(4, M), du=put(M, K), dr=put(M, K),
                                                 dparams=put(5, K), workspace=room)),
    "loss": (dq.dqrm_softmax_xent_fwd, dict(x=put(M, K), w=put(V, K), targets=put(M, dtype=torch.int64), loss=put(M), lse=put(M), bias=put(V), workspace=room)),
    "loss_bwd": (dq.dqrm_softmax_xent_bwd, dict(x=put(M, K), w=put(V, K), targets=put(M, dtype=torch.int64), lse=put(M), grad=put(M), dx=put(M, K), dw=put(V, K),
                                                dbias=put(V), bias=put(V), workspace=room)),
    "grad_norm": (dq.dqrm_grad_norm, dict(norm=put(1), grads=tensors, norms=put(2), workspace=room)),
    "grad_scale": (dq.dqrm_grad_scale, dict(norm=put(1), grads=tensors)),
    "grad_clip": (dq.dqrm_grad_clip, dict(norm=put(1), grads=tensors, norms=put(2), workspace=room)),
}


def make(call, gpus, **others):
    f, operands = OPERANDS[call]
    args = {name: how(gpus.get(name, gpus["all"])) for name, how in operands.items()}
    if call in ("grad_scale", "grad_clip"):
        args["max_norm"] = 1.0
    f(**args, **others)


@pytest.mark.parametrize("call", OPERANDS)
def test_an_operand_elsewhere_is_refused(call, library):
    for name in OPERANDS[call][1]:
        for where in (-1, 1):
            with pytest.raises(dq.DqrmError) as e:
                make(call, {"all": 0, name: where})
            assert e.value.code == dq.ERR_INVALID_ARG, (name, where)
    for others in ({}, dict(stream=0)):
        with pytest.raises(dq.DqrmError) as e:
            make(call, {"all": -1}, **others)
        assert e.value.code == dq.ERR_INVALID_ARG
    assert not library.calls


@pytest.mark.parametrize("call", OPERANDS)
def test_a_call_is_made_on_the_gpu_that_holds_its_operands(call, library):
    for current in (0, 1):
        for gpu in (0, 1, 3):
            library.current, library.calls = current, []
            make(call, {"all": gpu})
            make(call, {"all": gpu}, stream=77)
            assert [c[1:] for c in library.calls] == [(0 if gpu == 0 else 100 + gpu, gpu), (77, gpu)]
            assert library.current == current


def test_gradients_in_parts_on_two_devices():
    for tensors_, out, counts in (([put(4)(0), put(4)(1)], None, None), ([put(4, 2)(0)], [put(4, 2)(1)], None),
                                  ([put(4, 2)(0)], None, {0: put(1, dtype=torch.int32)(-1)})):
        with pytest.raises(dq.DqrmError) as e:
            dq.Grads(tensors_, out=out, counts=counts)
        assert e.value.code == dq.ERR_INVALID_ARG
    with pytest.raises(dq.DqrmError):
        dq.ResidualNorm(pre_gamma=put(K)(0), gate=put(K)(1))
