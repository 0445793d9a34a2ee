"""Host-side checks of svgear_linear, svgear_rotary and their backward passes that need no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2603_08982_amd as sv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_projection_argument_checks_are_clean_under_host_sanitizers(tmp_path_factory):
    """Every refusal and the workspace arithmetic, with the library's host code under AddressSanitizer and UBSan."""
    from paper_2603_08982_amd.build import HIPCC, build
    from test_sanitizers_cpu import ENV, SAN

    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not present")
    work = str(tmp_path_factory.mktemp("projection_san"))
    lib = build(lib=os.path.join(work, "libsvgear_san.so"), objdir=os.path.join(work, "obj"), host_sanitize=True)
    exe = os.path.join(work, "argcheck")
    clang = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "lib", "llvm", "bin", "clang")
    if not os.path.exists(clang):
        clang = "/opt/rocm/lib/llvm/bin/clang"
    cmd = [clang, *SAN, "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "native", "abi_argcheck_projections_main.c"), lib,
           "-Wl,-rpath," + work, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(ENV, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1"), timeout=300)
    assert r.returncode == 0, f"{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]
    assert "0 wrong result(s)" in r.stdout


def test_no_cpu_path():
    x, w = torch.zeros(2, 3, 4), torch.zeros(5, 4)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.linear(x, w)
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.linear_backward(torch.zeros(2, 3, 5), x, w)
    q = torch.zeros(1, 2, 3, 64)
    f = sv.rotary_frequencies((1, 1, 1), device="cpu")
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.rotary([q], f, (1, 1, 1), grid=(1, 1, 3))
    with pytest.raises(sv.SvgearError, match="device tensors"):
        sv.rotary_backward([q], None, f, (1, 1, 1), grid=(1, 1, 3))


def test_rotary_frequencies():
    f = sv.rotary_frequencies((2, 0, 3), theta=100.0, device="cpu")
    assert f.dtype == torch.float64
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3)], dtype=torch.float64), rtol=1e-15)


def test_workspaces_grow_with_what_is_copied():
    lib = sv.load_library()
    p = ctypes.c_void_p(0x10000)
    st = lambda b, n: (ctypes.c_int64 * 2)(b, n)
    size = lambda x, xst, w, ldw, dt=1: lib.svgear_linear_workspace(x, xst, w, ldw, dt, 2, 9000, 512, 2048)
    assert size(p, st(9000 * 512, 512), p, 512) == 0
    apart = size(p, st(9001 * 512, 512), p, 512)     # batches apart: x is copied
    assert apart >= 2 * 9000 * 512 * 2
    odd = size(ctypes.c_void_p(0x10002), st(9000 * 512, 512), p, 512)
    assert odd >= 2 * 9000 * 512 * 2
    both = size(p, st(9000 * 513, 513), p, 513)
    assert both >= (2 * 9000 + 2048) * 512 * 2
    assert size(p, st(9000 * 512, 512), p, 512, dt=7) == 0
