"""What the layer norm and dense attention refuse, without a GPU: the library's host code under sanitizers, and the Python entry
points in front of a library that must not be reached."""
import contextlib
import os
import subprocess

import pytest
import torch

import paper_2603_08982_amd as sv
from paper_2603_08982_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_argument_checks_are_clean_under_host_sanitizers(tmp_path_factory):
    """Every refusal and the workspace arithmetic, with the library's host code under AddressSanitizer and UBSan."""
    from paper_2603_08982_amd.build import HIPCC, build
    from test_sanitizers_cpu import ENV, SAN

    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not present")
    work = str(tmp_path_factory.mktemp("dense_san"))
    lib = build(lib=os.path.join(work, "libsvgear_san.so"), objdir=os.path.join(work, "obj"), host_sanitize=True)
    exe = os.path.join(work, "argcheck")
    clang = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "lib", "llvm", "bin", "clang")
    if not os.path.exists(clang):
        clang = "/opt/rocm/lib/llvm/bin/clang"
    cmd = [clang, *SAN, "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "native", "abi_argcheck_dense_main.c"), lib,
           "-Wl,-rpath," + work, "-lm", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(ENV, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1"), timeout=300)
    assert r.returncode == 0, f"{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]
    assert "0 wrong result(s)" in r.stdout


def test_no_cpu_path():
    x, q = torch.zeros(2, 3, 8), torch.zeros(1, 2, 3, 64)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.layer_norm(x)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.layer_norm_backward(x, x)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.attention(q, q, q)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.attention_backward(q, q, q, q, q, torch.zeros(1, 2, 3))


class Reached(Exception):
    pass


class NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                return 0
            raise Reached(name)

        return call


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(binding, "load_library", NoLibrary)
    monkeypatch.setattr(binding, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(binding, "_on_device", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(binding, "_stream_of", lambda device: 0)


BF, F, I = torch.bfloat16, torch.float32, torch.int32


def t(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


X = (2, 3, 16)
GOOD_NORM = {
    "alone": lambda: sv.layer_norm(t(*X)),
    "everything": lambda: sv.layer_norm(t(*X), t(16), t(16), scale=t(2, 16), shift=t(2, 16)),
    "of tokens": lambda: sv.layer_norm(t(*X), scale=t(*X), shift=t(*X)),
    "two dimensions": lambda: sv.layer_norm(t(3, 16), scale=t(16)),
    "strided": lambda: sv.layer_norm(t(2, 3, 32)[:, :, ::1][:, :, 5:21]),
    "backward": lambda: sv.layer_norm_backward(t(*X), t(*X), t(16), t(16), scale=t(2, 16), want=["dscale", "dx", "dweight", "dbias", "dshift"]),
}
BAD_NORM = {
    "another type": lambda: sv.layer_norm(t(*X), t(16, dtype=F)),
    "an unknown type": lambda: sv.layer_norm(t(*X, dtype=torch.float16)),
    "four dimensions": lambda: sv.layer_norm(t(1, 2, 3, 16)),
    "one dimension": lambda: sv.layer_norm(t(16)),
    "c not contiguous": lambda: sv.layer_norm(t(2, 16, 3).transpose(1, 2)),
    "no tokens": lambda: sv.layer_norm(t(2, 0, 16)),
    "c too long": lambda: sv.layer_norm(t(1, 1, (1 << 15) + 1)),
    "weight of another length": lambda: sv.layer_norm(t(*X), t(15)),
    "bias strided": lambda: sv.layer_norm(t(*X), None, t(32)[::2]),
    "scale of another batch": lambda: sv.layer_norm(t(*X), scale=t(3, 16)),
    "scale of one, shift of the other kind": lambda: sv.layer_norm(t(*X), scale=t(2, 16), shift=t(*X)),
    "shift strided": lambda: sv.layer_norm(t(*X), shift=t(2, 32)[:, ::2]),
    "negative eps": lambda: sv.layer_norm(t(*X), eps=-1.0),
    "eps that is none": lambda: sv.layer_norm(t(*X), eps=float("nan")),
    "out of another shape": lambda: sv.layer_norm(t(*X), out=t(2, 3, 17)),
    "out of another type": lambda: sv.layer_norm(t(*X), out=t(*X, dtype=F)),
    "dy of another shape": lambda: sv.layer_norm_backward(t(2, 4, 16), t(*X)),
    "nothing wanted": lambda: sv.layer_norm_backward(t(*X), t(*X), want=[]),
    "an unknown gradient": lambda: sv.layer_norm_backward(t(*X), t(*X), want=["dw"]),
    "dshift without a scale": lambda: sv.layer_norm_backward(t(*X), t(*X), want=["dshift"]),
}
Q, K = (2, 4, 10, 64), (2, 2, 7, 64)
L = (2, 4, 10)


def at(q=None, k=None, v=None, **kw):
    return sv.attention(t(*Q) if q is None else q, t(*K) if k is None else k, t(*K) if v is None else v, **kw)


def back(dy=None, o=None, lse=None, **kw):
    return sv.attention_backward(t(*Q) if dy is None else dy, t(*Q), t(*K), t(*K), t(*Q) if o is None else o,
                                 t(*L, dtype=F) if lse is None else lse, **kw)


GOOD_ATTENTION = {
    "alone": lambda: at(),
    "masks": lambda: at(causal=True, prefix=t(2, 3, dtype=I), q_offsets=t(2, 4, dtype=I), k_offsets=t(2, 4, dtype=I), cap=3.0, slopes=t(4, dtype=F)),
    "one row for the batch": lambda: at(causal=True, prefix=t(3, dtype=I), q_offsets=t(4, dtype=I), k_offsets=t(4, dtype=I)),
    "lengths": lambda: at(k_offsets=t(2, 2, dtype=I), want_lse=True),
    "backward": lambda: back(),
    "backward of the keys": lambda: back(want=["dk", "dv"], out={"dv": t(*K)}),
}
BAD_ATTENTION = {
    "another type": lambda: at(k=t(*K, dtype=F)),
    "an unknown type": lambda: at(t(*Q, dtype=torch.float16), t(*K, dtype=torch.float16), t(*K, dtype=torch.float16)),
    "three dimensions": lambda: at(q=t(4, 10, 64)),
    "d of 32": lambda: at(t(2, 4, 10, 32), t(2, 2, 7, 32), t(2, 2, 7, 32)),
    "d of k another": lambda: at(k=t(2, 2, 7, 128), v=t(2, 2, 7, 128)),
    "v of other keys": lambda: at(v=t(2, 2, 8, 64)),
    "another batch": lambda: at(k=t(3, 2, 7, 64), v=t(3, 2, 7, 64)),
    "heads that do not divide": lambda: at(k=t(2, 3, 7, 64), v=t(2, 3, 7, 64)),
    "no keys": lambda: at(k=t(2, 2, 0, 64), v=t(2, 2, 0, 64)),
    "no queries": lambda: at(q=t(2, 4, 0, 64)),
    "d not contiguous": lambda: at(q=t(2, 4, 64, 10).transpose(2, 3)),
    "slopes of other heads": lambda: at(slopes=t(3, dtype=F)),
    "slopes of another type": lambda: at(slopes=t(4)),
    "prefix without causal": lambda: at(prefix=t(2, 1, dtype=I)),
    "prefix of another shape": lambda: at(causal=True, prefix=t(2, 2, dtype=I)),
    "offsets of another type": lambda: at(k_offsets=t(2, 2, dtype=torch.int64)),
    "offsets of another batch": lambda: at(k_offsets=t(3, 2, dtype=I)),
    "offsets of one entry": lambda: at(k_offsets=t(2, 1, dtype=I)),
    "several documents of the keys alone": lambda: at(k_offsets=t(2, 4, dtype=I)),
    "offsets of other documents": lambda: at(q_offsets=t(2, 3, dtype=I), k_offsets=t(2, 4, dtype=I)),
    "offsets of one and of each": lambda: at(q_offsets=t(3, dtype=I), k_offsets=t(2, 3, dtype=I)),
    "offsets strided": lambda: at(k_offsets=t(2, 4, dtype=I)[:, ::2]),
    "negative cap": lambda: at(cap=-2.0),
    "infinite scale": lambda: at(scale=float("inf")),
    "out of another shape": lambda: at(out=t(2, 4, 11, 64)),
    "out of another type": lambda: at(out=t(*Q, dtype=F)),
    "dy of another shape": lambda: back(dy=t(2, 4, 11, 64)),
    "lse of another type": lambda: back(lse=t(*L)),
    "lse of another shape": lambda: back(lse=t(2, 4, 11, dtype=F)),
    "dk alone": lambda: back(want=["dk"]),
    "nothing wanted": lambda: back(want=[]),
    "an unknown gradient": lambda: back(want=["dslopes"]),
    "an output that is not wanted": lambda: back(want=["dq"], out={"dk": t(*K)}),
    "an output of another shape": lambda: back(out={"dq": t(*K)}),
}


@pytest.mark.parametrize("what", [*GOOD_NORM, *(f"attention {n}" for n in GOOD_ATTENTION)])
def test_good_calls_reach_the_library(no_library, what):
    with pytest.raises(Reached):
        (GOOD_ATTENTION[what[10:]] if what.startswith("attention ") else GOOD_NORM[what])()


@pytest.mark.parametrize("what", BAD_NORM)
def test_layer_norm_refuses(no_library, what):
    with pytest.raises(sv.SvgearError):
        BAD_NORM[what]()


@pytest.mark.parametrize("what", BAD_ATTENTION)
def test_attention_refuses(no_library, what):
    with pytest.raises(sv.SvgearError):
        BAD_ATTENTION[what]()


def test_the_shift_of_a_gradient(no_library):
    """dshift takes its shape from the scale or, without one, from the shift; dscale needs the scale."""
    for kw in ({"shift": t(2, 16)}, {"shift": t(*X)}, {"scale": t(2, 16), "shift": t(2, 16)}):
        with pytest.raises(Reached):
            sv.layer_norm_backward(t(*X), t(*X), want=["dshift", "dx"], **kw)
    for kw in ({"shift": t(3, 16)}, {"shift": t(2, 16, dtype=F)}, {"scale": t(*X), "shift": t(2, 16)}, {"shift": t(2, 32)[:, ::2]}):
        with pytest.raises(sv.SvgearError):
            sv.layer_norm_backward(t(*X), t(*X), want=["dshift"], **kw)
    with pytest.raises(sv.SvgearError, match="dscale"):
        sv.layer_norm_backward(t(*X), t(*X), want=["dscale"], shift=t(2, 16))


BLOCK = {"x": (2, 3, 16), "context": (2, 5, 24), "w_q": (128, 16), "w_kv": (256, 24), "w_out": (16, 128), "heads": 2}


def block(**change):
    a = {n: t(*v) if isinstance(v, tuple) else v for n, v in {**BLOCK, **change}.items()}
    return sv.cross_attention_block(**a)


def test_cross_attention_block_reaches_the_library(no_library):
    with pytest.raises(Reached):
        block()


@pytest.mark.parametrize("change", [{"w_q": (0, 16)}, {"w_kv": (0, 24)}, {"w_q": (129, 16)}, {"w_kv": (200, 24)}, {"w_out": (16, 64)}, {"heads": 0},
                                    {"heads": -1}, {"x": (3, 16)}, {"context": (1, 5, 24)}, {"w_q": (128,)}, {"w_out": (128,)}], ids=str)
def test_cross_attention_block_refuses(no_library, change):
    with pytest.raises(sv.SvgearError):
        block(**change)


@pytest.mark.parametrize("kw", [{"cap": 1e-46}, {"cap": 1e-40}, {"cap": float("inf")}, {"cap": float("nan")}, {"cap": -0.5}], ids=str)
def test_caps_that_fp32_has_not(no_library, kw):
    with pytest.raises(sv.SvgearError):
        at(**kw)
    with pytest.raises(sv.SvgearError):
        back(**kw)


@pytest.mark.parametrize("scale,cap", [(3e38, 0.0), (-3e38, 0.0), (0.125, 3e38), (1e10, 1e-37), (-1e10, 1e-37), (1e-8, 1e37), (1e-45, 1.0), (3e38, 1e38)])
def test_factors_that_fp32_has_not(scale, cap):
    """scale log2(e), cap log2(e) and scale / cap have to be numbers of fp32: refused by the library, in front of all that touches a device."""
    import ctypes

    lib = sv.load_library()
    stride = lambda *n: (ctypes.c_int64 * 3)(*n)
    q, k, sizes = stride(25600, 6400, 64), stride(6400, 3200, 64), (1, 2, 4, 2, 100, 50, 64)
    p = [0x10000 * (i + 1) for i in range(12)]
    mask = (scale, cap, None, 0, 0, None, None, None)
    assert lib.svgear_attention(p[0], q, p[1], k, p[2], k, *sizes, *mask, p[3], q, None, p[4], 1 << 40, None) == -1
    assert lib.svgear_attention_backward(p[0], q, p[1], q, p[2], k, p[3], k, p[4], q, p[5], *sizes, *mask, p[6], q, p[7], k, p[8], k, p[9], 1 << 40,
                                         None) == -1
