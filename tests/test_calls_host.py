"""The compiled part of the binding: how it takes its arguments, and that it keeps no reference to them."""
import sys

import numpy as np
import pytest

from paper_2605_28803_gb300 import qvla

CALLS = ["qvla_fp4_quantize_rows", "qvla_fp4_dequantize_rows", "qvla_gemm_fp4", "qvla_fp4_linear", "qvla_block_norm", "qvla_block_norm_fp4"]


class Address:
    """Stands for a tensor: an address that the refused calls below never read."""

    def __init__(self, value=1 << 20):
        self.value = value

    def data_ptr(self):
        return self.value


def rows(**changes):
    args = dict(x=Address(), xdt=qvla.BF16, x_stride=128, M=1, K=128, had_block=1, fmt=qvla.MXFP4, step_scale=None, xq=Address(), xs=Address())
    args.update(changes)
    return args


@pytest.mark.parametrize("call", CALLS)
def test_a_call_without_arguments_names_the_first_missing_one(call):
    with pytest.raises(TypeError, match=f"{call}\\(\\) needs the argument"):
        getattr(qvla, call)()


@pytest.mark.parametrize("call", CALLS)
def test_too_many_unknown_and_repeated_arguments(call):
    f = getattr(qvla, call)
    with pytest.raises(TypeError, match="arguments but 40 were given"):
        f(*[None] * 40)
    with pytest.raises(TypeError, match="no argument 'nonsense'"):
        f(nonsense=1)
    with pytest.raises(TypeError, match="two values for argument"):
        first = f.__text_signature__.strip("()").split(",")[0]
        f(None, **{first: None})


@pytest.mark.parametrize("changes, error", [
    (dict(M="1"), TypeError), (dict(M=1.0), TypeError), (dict(M=1 << 31), OverflowError), (dict(K=-(1 << 31) - 1), OverflowError),
    (dict(x_stride=1 << 63), OverflowError), (dict(x=3), AttributeError), (dict(x=Address("text")), TypeError), (dict(stream="s"), AttributeError),
    (dict(xscale=Address(1 << 70)), OverflowError)])
def test_arguments_of_the_wrong_kind(changes, error):
    with pytest.raises(error):
        qvla.qvla_fp4_quantize_rows(**rows(**changes))


def test_the_librarys_own_refusals_arrive_as_its_errors():
    with pytest.raises(qvla.QvlaError):
        qvla.qvla_fp4_quantize_rows(**rows(K=63))
    with pytest.raises(qvla.QvlaError):
        qvla.qvla_fp4_quantize_rows(**rows(x=None))
    qvla.qvla_fp4_quantize_rows(**rows(M=np.int64(0), K=np.int32(128), x_stride=np.int64(128)))  # no rows: nothing is launched


def test_no_reference_is_kept():
    x, stride = Address(), 123456789
    before = sys.getrefcount(x), sys.getrefcount(stride)
    for _ in range(100):
        with pytest.raises(qvla.QvlaError):
            qvla.qvla_fp4_quantize_rows(**rows(x=x, xs=x, K=63, x_stride=stride))
        with pytest.raises(TypeError):
            qvla.qvla_fp4_quantize_rows(x, nonsense=x)
        with pytest.raises(TypeError):
            qvla.qvla_fp4_quantize_rows(**rows(x=x, M="1"))
    assert (sys.getrefcount(x), sys.getrefcount(stride)) == before


def norm(**vectors):
    return qvla.BlockNorm(qvla.NORM_RMS, qvla.BF16, **vectors)


def junction(n, K=128, M=0):
    """Without rows nothing is launched."""
    qvla.qvla_block_norm(n, Address(), qvla.BF16, K, None, 0, M, K, None, Address())
    qvla.qvla_block_norm_fp4(n, Address(), qvla.BF16, K, None, 0, M, K, None, None, 1, qvla.MXFP4, None, Address(), Address())


def test_norms_whose_vectors_do_not_fit():
    torch = pytest.importorskip("torch")

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)

    junction(norm(post_norm=True, post_weight=t(128), pre_weight=t(128), pre_bias=t(256), gate=t(2, 128), mod_tokens=1))
    for vectors in (dict(pre_weight=t(64)), dict(pre_weight=t(128), pre_bias=t(120)), dict(post_norm=True, post_weight=t(127)), dict(scale=t(2, 64), mod_tokens=1)):
        with pytest.raises(ValueError, match="channels"):
            junction(norm(**vectors))
    index = dict(gate=t(2, 128), mod_index=t(5, dtype=torch.int32))
    junction(norm(**index))
    for call, args in ((qvla.qvla_block_norm, (None, Address())),
                       (qvla.qvla_block_norm_fp4, (None, None, 1, qvla.MXFP4, None, Address(), Address()))):
        with pytest.raises(ValueError, match="mod_index has 5 tokens, the call 6"):
            call(norm(**index), Address(), qvla.BF16, 128, None, 0, 6, 128, *args)
    for vectors in (dict(pre_weight=t(128, dtype=torch.float32)), dict(pre_bias=t(128, dtype=torch.float16)), dict(pre_weight=t(1, 128)),
                    dict(pre_weight=t(256)[::2]), dict(gate=t(2, 128, dtype=torch.float32)), dict(gate=t(2, 128), mod_index=t(5, dtype=torch.int64)),
                    dict(gate=t(2, 128), mod_index=t(10, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            norm(**vectors)


def test_objects_of_another_kind():
    class Handle:
        handle, ref, dt, width, tokens = 1 << 20, 1 << 20, 0, 1 << 20, 1 << 20

    for call, args in ((qvla.qvla_gemm_fp4, (Address(), Address(), None, 1, Address())), (qvla.qvla_fp4_linear, (Address(), 1, None, Address(), Address(), 0))):
        for other in (Handle(), None, 1 << 20):
            with pytest.raises(TypeError, match="an Fp4Layer is needed"):
                call(other, *args)
    with pytest.raises(TypeError, match="a BlockNorm is needed"):
        junction(Handle())
    closed = qvla.Fp4Layer(None, 128, 128, 1, qvla.MXFP4, qvla.BF16, qvla.BF16, False)
    with pytest.raises(qvla.QvlaError, match="layer must not be NULL"):
        qvla.qvla_gemm_fp4(closed, Address(), Address(), None, 1, Address())


def test_the_compiled_part_alone_refuses_calls():
    """Without the rest of the binding it knows no types and no errors."""
    import subprocess

    run = subprocess.run([sys.executable, "-c", "\n".join([
        "import importlib.util, sys",
        f"spec = importlib.util.spec_from_file_location('_calls', {qvla._calls.__file__!r})",
        "m = importlib.util.module_from_spec(spec); spec.loader.exec_module(m)",
        "for call in ('qvla_gemm_fp4', 'qvla_block_norm', 'qvla_fp4_quantize_rows'):",
        "    try:",
        "        getattr(m, call)(*[None] * {'qvla_gemm_fp4': 7, 'qvla_block_norm': 11, 'qvla_fp4_quantize_rows': 12}[call])",
        "    except RuntimeError as e:",
        "        print(e)"])], capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout.count("not set up") == 3, run.stderr
