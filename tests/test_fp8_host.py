"""The 8-bit operators' refusals and marshalling; no GPU needed."""
import copyreg
import ctypes
import importlib.machinery
import importlib.util
import inspect
import os
import pickle
import re

import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc
from paper_2312_17482_amd import binding as mb
from paper_2312_17482_amd import build
from tests.test_lds_load import assembly, too_early
from tests.test_marshal import STREAM, c_parameters

lib = mb.raw()
A = 4096            # a fake, 16-byte aligned "device pointer": must never be dereferenced by these calls
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BAD, NOT = mb.MB_ERR_INVALID_ARG, mb.MB_ERR_UNSUPPORTED

GOOD = {
    "mb_fp8_quant": dict(x=A, x_row_stride=144, T_cap=5, meta_dev=None, W=144, dt=mb.MB_BF16, q=A, s=A, stream=None),
    "mb_fp8_dequant": dict(q=A, s=A, T_cap=5, meta_dev=None, W=144, dt=mb.MB_F32, x=A, x_row_stride=144, stream=None),
    "mb_fp8_quant_weight": dict(w=A, n_out=80, n_in=144, dt=mb.MB_F32, q=A, s=A, qt=A, st=A, stream=None),
    "mb_linear_fp8_fwd": dict(xq=A, xs=A, wq=A, ws=A, T_cap=5, meta_dev=None, n_in=144, n_out=80, dt=mb.MB_BF16, y=A, y_row_stride=80,
                              stream=None),
    "mb_linear_fp8_wgrad": dict(dy=A, dys=None, dy_row_stride=80, xq=A, xs=A, T_cap=5, meta_dev=None, n_in=144, n_out=80, dw=A,
                                workspace=None, workspace_bytes=0, stream=None),
    "mb_geglu_fp8_act": dict(xq=A, xs=A, w1vq=A, w1vs=A, T_cap=5, meta_dev=None, hidden=144, inter=256, actq=A, acts=A, stream=None),
    "mb_gelu_gate_fp8_bwd": dict(da=A, hg=A, hgs=A, T_cap=5, meta_dev=None, inter=256, dhgq=A, dhgs=A, stream=None),
}
REFUSED = [
    ("mb_fp8_quant", dict(W=0), BAD, "positive"), ("mb_fp8_quant", dict(W=24), NOT, "multiple of 16"),
    ("mb_fp8_quant", dict(W=1 << 21), NOT, "2^20"), ("mb_fp8_quant", dict(T_cap=-1), BAD, "T_cap"),
    ("mb_fp8_quant", dict(T_cap=(1 << 30) + 1), NOT, "2^30"), ("mb_fp8_quant", dict(dt=7), BAD, "dtype"),
    ("mb_fp8_quant", dict(x_row_stride=128), BAD, "x_row_stride"), ("mb_fp8_quant", dict(x_row_stride=148), BAD, "16 bytes"),
    ("mb_fp8_quant", dict(x_row_stride=1 << 21), NOT, "2^21"), ("mb_fp8_quant", dict(x=A + 8), BAD, "x is not 16-byte"),
    ("mb_fp8_quant", dict(q=None), BAD, "q is NULL"), ("mb_fp8_quant", dict(s=None), BAD, "s is NULL"),
    ("mb_fp8_dequant", dict(W=40), NOT, "multiple of 16"), ("mb_fp8_dequant", dict(x=None), BAD, "x is NULL"),
    ("mb_fp8_dequant", dict(x_row_stride=146), BAD, "16 bytes"), ("mb_fp8_dequant", dict(q=A + 1), BAD, "q is not"),
    ("mb_fp8_quant_weight", dict(n_out=8), NOT, "n_out"), ("mb_fp8_quant_weight", dict(n_in=-16), BAD, "n_in"),
    ("mb_fp8_quant_weight", dict(qt=None), BAD, "together"), ("mb_fp8_quant_weight", dict(st=None), BAD, "together"),
    ("mb_fp8_quant_weight", dict(w=None), BAD, "w is NULL"), ("mb_fp8_quant_weight", dict(qt=A + 4), BAD, "qt is not"),
    ("mb_linear_fp8_fwd", dict(n_in=72), NOT, "n_in"), ("mb_linear_fp8_fwd", dict(n_out=8), NOT, "n_out"),
    ("mb_linear_fp8_fwd", dict(y_row_stride=64), BAD, "y_row_stride"), ("mb_linear_fp8_fwd", dict(y_row_stride=84), BAD, "16 bytes"),
    ("mb_linear_fp8_fwd", dict(y_row_stride=1 << 22), NOT, "2^21"), ("mb_linear_fp8_fwd", dict(ws=None), BAD, "ws is NULL"),
    ("mb_linear_fp8_fwd", dict(T_cap=1 << 30, n_out=1 << 10, y_row_stride=1 << 10), NOT, "2^38"),
    ("mb_linear_fp8_fwd", dict(xs=A + 2), BAD, "xs is not"), ("mb_linear_fp8_fwd", dict(y=None), BAD, "y is NULL"),
    ("mb_linear_fp8_wgrad", dict(dw=None), BAD, "dw is NULL"), ("mb_linear_fp8_wgrad", dict(dy=None), BAD, "dy is NULL"),
    ("mb_linear_fp8_wgrad", dict(dys=A, dy_row_stride=96), BAD, "contiguous"), ("mb_linear_fp8_wgrad", dict(dys=A + 2), BAD, "dys is not"),
    ("mb_linear_fp8_wgrad", dict(dy_row_stride=72), BAD, "dy_row_stride"), ("mb_linear_fp8_wgrad", dict(xq=None), BAD, "xq is NULL"),
    ("mb_linear_fp8_wgrad", dict(T_cap=27000), mb.MB_ERR_WORKSPACE, "needed"),
    ("mb_fp8_quant", dict(T_cap=1 << 29, W=16, x_row_stride=16), NOT, "2^29"), ("mb_fp8_dequant", dict(T_cap=1 << 30, W=16, x_row_stride=16), NOT, "2^29"),
    ("mb_linear_fp8_wgrad", dict(n_in=1 << 16, n_out=1 << 15, dy_row_stride=1 << 15), NOT, "gradient of 2^31"),
    ("mb_linear_fp8_wgrad", dict(T_cap=27000, workspace=A + 8, workspace_bytes=1 << 30), BAD, "workspace is not"),
    ("mb_geglu_fp8_act", dict(inter=192), NOT, "multiple of 128"), ("mb_geglu_fp8_act", dict(hidden=8), NOT, "hidden"),
    ("mb_geglu_fp8_act", dict(hidden=1 << 16, inter=1 << 16), NOT, "2^31"), ("mb_geglu_fp8_act", dict(acts=None), BAD, "acts is NULL"),
    ("mb_gelu_gate_fp8_bwd", dict(inter=64), NOT, "multiple of 128"), ("mb_gelu_gate_fp8_bwd", dict(hgs=A + 8), BAD, "hgs is not"),
    ("mb_gelu_gate_fp8_bwd", dict(da=None), BAD, "da is NULL"), ("mb_gelu_gate_fp8_bwd", dict(dhgs=None), BAD, "dhgs is NULL"),
]


@pytest.mark.parametrize("name,over,status,needle", REFUSED)
def test_refused_without_launching(name, over, status, needle):
    args = dict(GOOD[name], **over)
    assert list(args) == c_parameters(name)
    assert getattr(lib, name)(*args.values()) == status
    assert needle in mb.mb_last_error()


@pytest.mark.parametrize("name", [n for n in GOOD if "T_cap" in GOOD[n] and n != "mb_linear_fp8_wgrad"])
def test_no_rows_need_no_gpu(name):
    args = {k: None if v == A else v for k, v in GOOD[name].items()}
    assert getattr(lib, name)(*dict(args, T_cap=0).values()) == mb.MB_OK


def test_workspace_sizes():
    assert mb.mb_linear_fp8_wgrad_workspace_bytes(64, 768, 768) == 0 == mb.mb_linear_fp8_wgrad_workspace_bytes(-1, 768, 768)
    need = mb.mb_linear_fp8_wgrad_workspace_bytes(26963, 768, 768)
    assert need % (4 * 768 * 768) == 0 and need >= 2 * 4 * 768 * 768


# ---------------------------------------------------------------------------------------------------- marshalling
NATIVE = [n for n in GOOD]


@pytest.fixture
def recorded():
    """The native 8-bit calls with a C ABI of this test's: (calls, what each was handed last)."""
    loader = importlib.machinery.ExtensionFileLoader("_mosaic_marshal", mb._MARSHAL_PATH)
    native = importlib.util.module_from_spec(importlib.util.spec_from_loader("_mosaic_marshal", loader))
    loader.exec_module(native)
    seen, kept, addresses = {}, [], {"mb_last_error": ctypes.cast(lib.mb_last_error, ctypes.c_void_p).value}

    def stand_in(name):
        real, names = getattr(lib, name), c_parameters(name)
        assert len(names) == len(real.argtypes)

        def f(*args):
            seen[name] = dict(zip(names, args))
            return 1000 if name.endswith("_bytes") else mb.MB_OK
        kept.append(ctypes.CFUNCTYPE(real.restype, *real.argtypes)(f))
        addresses[name] = ctypes.cast(kept[-1], ctypes.c_void_p).value
    for name in NATIVE + ["mb_linear_fp8_wgrad_workspace_bytes"]:
        stand_in(name)
    yield native.Fp8Calls(addresses, mb.MosaicAttnError, lambda: 3, lambda device: STREAM + device, None), seen
    with pytest.raises(KeyError):
        native.Fp8Calls({k: v for k, v in addresses.items() if k != "mb_fp8_quant"}, mb.MosaicAttnError, None, None, None)
    del kept


def eight(rows, W, block=1):
    return torch.zeros(rows, W).to(E4M3), torch.zeros(-(-rows // block), -(-W // 128), dtype=torch.uint8).view(E8M0)


def meta():
    return torch.zeros(2, dtype=torch.int32)


def all_arguments():
    """name -> (arguments in their documented order, what else the C function has to be handed)."""
    bf = torch.bfloat16
    T, W, N, I = 9, 144, 272, 256
    wide = lambda cols, dtype=bf: torch.zeros(T, 2 * cols, dtype=dtype)[:, :cols]
    xq, xs = eight(T, W)
    wq, ws = eight(N, W, 128)
    q, s = eight(T, W)
    yield "mb_fp8_quant", dict(x=wide(W), T_cap=4, meta=meta(), q=q, s=s), dict(x_row_stride=2 * W, W=W, dt=mb.MB_BF16)
    yield "mb_fp8_dequant", dict(q=xq, s=xs, dtype=torch.float32, T_cap=4, meta=meta(), out=wide(W, torch.float32)), dict(
        x_row_stride=2 * W, W=W, dt=mb.MB_F32)
    qt, st = eight(W, N, 128)
    yield "mb_fp8_quant_weight", dict(w=torch.zeros(N, W), transposed=True, q=wq, s=ws, qt=qt, st=st), dict(
        n_out=N, n_in=W, dt=mb.MB_F32)
    yield "mb_linear_fp8_fwd", dict(xq=xq, xs=xs, wq=wq, ws=ws, dtype=bf, T_cap=4, meta=meta(), y=wide(N)), dict(
        n_in=W, n_out=N, dt=mb.MB_BF16, y_row_stride=2 * N)
    dy, dys = eight(T, N)
    yield "mb_linear_fp8_wgrad", dict(dy=dy, xq=xq, xs=xs, dys=dys, T_cap=4, meta=meta(), dw=torch.zeros(N, W),
                                      workspace=torch.zeros(33, dtype=torch.uint8)), dict(
        dy_row_stride=N, n_in=W, n_out=N, workspace_bytes=33)
    w1vq, w1vs = eight(2 * I, W, 128)
    aq, asc = eight(T, I)
    yield "mb_geglu_fp8_act", dict(xq=xq, xs=xs, w1vq=w1vq, w1vs=w1vs, T_cap=4, meta=meta(), actq=aq, acts=asc), dict(hidden=W, inter=I)
    hg, hgs = eight(T, 2 * I)
    dhg, dhgs = eight(T, 2 * I)
    yield "mb_gelu_gate_fp8_bwd", dict(da=torch.zeros(T, I, dtype=bf), hg=hg, hgs=hgs, T_cap=4, meta=meta(), dhgq=dhg, dhgs=dhgs), dict(
        inter=I)


RENAMED = {"meta": "meta_dev", "out": "x"}


@pytest.mark.parametrize("by_name", [False, True])
def test_every_argument_arrives(recorded, by_name):
    calls, seen = recorded
    for name, args, rest in all_arguments():
        result = getattr(calls, name)(**args) if by_name else getattr(calls, name)(*args.values())
        got = seen[name]
        want = {RENAMED.get(k, k): v.data_ptr() if isinstance(v, torch.Tensor) else v for k, v in args.items()}
        want = {k: v for k, v in want.items() if k in got}
        want.update(rest, stream=STREAM + 3)
        assert got == want, name
        outputs = [v for k, v in args.items() if k in ("q", "s", "qt", "st", "out", "y", "dw", "actq", "acts", "dhgq", "dhgs")]
        if name == "mb_fp8_dequant":
            outputs = [args["out"]]
        result = result if isinstance(result, tuple) else (result,)
        assert len(result) == len(outputs) and all(a is b for a, b in zip(result, outputs)), name


def test_defaults(recorded):
    calls, seen = recorded
    x = torch.zeros(5, 144)
    q, s = calls.mb_fp8_quant(x)
    assert (q.dtype, q.shape, s.dtype, s.shape) == (E4M3, (5, 144), E8M0, (5, 2))
    assert seen["mb_fp8_quant"]["T_cap"] == 5 and seen["mb_fp8_quant"]["x_row_stride"] == 144 and seen["mb_fp8_quant"]["dt"] == mb.MB_F32
    assert calls.mb_fp8_dequant(q, s).dtype == torch.bfloat16
    w = torch.zeros(272, 144, dtype=torch.bfloat16)
    wq, ws, qt, st = calls.mb_fp8_quant_weight(w)
    assert [t.shape for t in (wq, ws, qt, st)] == [(272, 144), (3, 2), (144, 272), (2, 3)]
    assert len(calls.mb_fp8_quant_weight(w, transposed=False)) == 2
    assert seen["mb_fp8_quant_weight"]["qt"] is None is seen["mb_fp8_quant_weight"]["st"]
    y = calls.mb_linear_fp8_fwd(q, s, wq, ws)
    assert (y.dtype, y.shape) == (torch.bfloat16, (5, 272)) and seen["mb_linear_fp8_fwd"]["meta_dev"] is None
    assert calls.mb_linear_fp8_fwd(q, s, wq, ws, dtype=torch.float32).dtype == torch.float32
    dw = calls.mb_linear_fp8_wgrad(y, q, s)
    assert (dw.dtype, dw.shape) == (torch.float32, (272, 144))
    assert seen["mb_linear_fp8_wgrad"]["dys"] is None and seen["mb_linear_fp8_wgrad"]["workspace_bytes"] == 1000
    w1vq, w1vs = eight(512, 144, 128)
    aq, asc = calls.mb_geglu_fp8_act(q, s, w1vq, w1vs)
    assert aq.shape == (5, 256) and asc.shape == (5, 2)
    dq, ds = calls.mb_gelu_gate_fp8_bwd(torch.zeros(5, 256, dtype=torch.bfloat16), torch.zeros(5, 512, dtype=torch.bfloat16))
    assert dq.shape == (5, 512) and ds.shape == (5, 4) and seen["mb_gelu_gate_fp8_bwd"]["hgs"] is None


def test_shapes_that_do_not_fit_are_refused(recorded):
    calls, seen = recorded
    xq, xs = eight(5, 144)
    wq, ws = eight(272, 144, 128)
    bf = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)
    wrong = [
        lambda: calls.mb_fp8_quant(torch.zeros(5, 144).t()), lambda: calls.mb_fp8_quant(torch.zeros(5)),
        lambda: calls.mb_fp8_quant(torch.zeros(5, 144), T_cap=6), lambda: calls.mb_fp8_quant(torch.zeros(5, 144), q=xq, s=xs[:4]),
        lambda: calls.mb_fp8_quant(torch.zeros(6, 144), q=xq, s=xs), lambda: calls.mb_fp8_quant(torch.zeros(5, 128), q=xq, s=xs),
        lambda: calls.mb_fp8_dequant(xq, xs[:, :1]), lambda: calls.mb_fp8_dequant(xq.view(torch.uint8), xs),
        lambda: calls.mb_fp8_dequant(xq, xs, out=bf(4, 144)), lambda: calls.mb_fp8_dequant(xq, xs, torch.float32, out=bf(5, 144)),
        lambda: calls.mb_fp8_quant_weight(torch.zeros(144, 272).t()), lambda: calls.mb_fp8_quant_weight(torch.zeros(272, 144), False, qt=wq, st=ws),
        lambda: calls.mb_fp8_quant_weight(torch.zeros(272, 144), qt=wq, st=ws),
        lambda: calls.mb_linear_fp8_fwd(xq, xs, *eight(272, 128, 128)), lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, xs),
        lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, ws, y=bf(5, 256)), lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, ws, y=bf(4, 272)),
        lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, ws, y=bf(272, 5).t()), lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, ws, torch.float32, y=bf(5, 272)),
        lambda: calls.mb_linear_fp8_wgrad(bf(4, 272), xq, xs), lambda: calls.mb_linear_fp8_wgrad(torch.zeros(5, 272), xq, xs),
        lambda: calls.mb_linear_fp8_wgrad(bf(5, 272), xq, xs, dw=torch.zeros(144, 272)), lambda: calls.mb_linear_fp8_wgrad(xq, xq, xs, dys=xs[:4]),
        lambda: calls.mb_geglu_fp8_act(xq, xs, *eight(512, 128, 128)),
        lambda: calls.mb_gelu_gate_fp8_bwd(bf(5, 256), bf(5, 256)), lambda: calls.mb_gelu_gate_fp8_bwd(bf(5, 256), bf(4, 512)),
        lambda: calls.mb_gelu_gate_fp8_bwd(torch.zeros(5, 256), bf(5, 512)),
        lambda: calls.mb_linear_fp8_fwd(xq, xs, wq.to("meta"), ws),
    ]
    seen.clear()
    for i, call in enumerate(wrong):
        with pytest.raises(AssertionError):
            call()
            print("call", i)
    for call in (lambda: calls.mb_fp8_quant(torch.zeros(5, 144, dtype=torch.float16)), lambda: calls.mb_fp8_dequant(xq, xs, "float32"),
                 lambda: calls.mb_linear_fp8_fwd(xq, xs, wq, ws, torch.float16), lambda: calls.mb_linear_fp8_fwd(xq, xs, wq),
                 lambda: calls.mb_fp8_quant(torch.zeros(5, 144), rows=4)):
        with pytest.raises(TypeError):
            call()
    assert not [k for k in seen if not k.endswith("_bytes")]


def test_the_calls_pickle_by_name_and_say_what_they_take():
    for name in NATIVE:
        f = getattr(mb, name)
        assert pickle.loads(pickle.dumps(f)) == f
        assert list(inspect.signature(f).parameters) == list(next(a for n, a, _ in all_arguments() if n == name))
        assert f.__doc__


def test_no_byte_load_comes_too_early(tmp_path):
    """Loads of bytes into LDS need the wait states of those of words, in front of them."""
    code = assembly(os.path.join(build.CSRC, "fp8_gemm.hip"), tmp_path / "code.s")
    words, _ = too_early(code)
    loads, found = too_early([re.sub("buffer_load_ubyte (.* lds)$", r"buffer_load_dword \1", l) for l in code])
    assert loads > words > 0 and not found, found[:10]


# ---------------------------------------------------------------------------------------------------- the oracle
def test_oracle_rounding_is_the_nearest_code():
    """Against the table of all codes, ties to the even one."""
    codes = orc.e4m3_values()
    pos = codes[:127]
    assert np.all(np.diff(pos) > 0) and pos[-1] == 448.0 and np.isnan(codes[127])
    x = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 4000), np.ldexp(np.random.default_rng(1).uniform(-1, 1, 4000), -6),
                        pos, (pos[1:] + pos[:-1]) / 2, -(pos[1:] + pos[:-1]) / 2])
    d = np.abs(np.abs(x)[:, None] - pos[None, :])
    near = d.argmin(1)
    tie = np.isclose(d[np.arange(len(x)), near], d[np.arange(len(x)), np.minimum(near + 1, 126)], rtol=0, atol=0) & (near < 126)
    want = np.where(tie & (near % 2 == 1), pos[np.minimum(near + 1, 126)], pos[near])
    assert np.array_equal(np.abs(orc.round_e4m3(x)), want)


def test_oracle_scales_are_the_smallest_that_hold():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((50, 300)) * np.exp(5 * rng.standard_normal((50, 1)))
    x[0], x[1, :128] = 0.0, 448.0
    q, e = orc.store(x)
    for i in range(50):
        for j in range(3):
            top = np.abs(x[i, j * 128:(j + 1) * 128]).max()
            assert top <= np.ldexp(448.0, e[i, j]) and (e[i, j] == -126 or top > np.ldexp(448.0, e[i, j] - 1))
    assert np.all(np.abs(orc.values(q, e) - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * np.repeat(np.ldexp(1.0, e), 128, 1)[:, :300])
