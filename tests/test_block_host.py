"""Host side of the transformer-block operators (CPU): argument checks that come before any launch, workspaces,
struct layouts, and the failure of a launch without a device."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2607_12505_amd import build, nmblock, nmspmm

FAKE, NUL = 1 << 20, None
ARG, SHAPE, WS, HIP, UNSUPPORTED = (nmspmm.NM_ERR_ARG, nmspmm.NM_ERR_SHAPE, nmspmm.NM_ERR_WORKSPACE,
                                    nmspmm.NM_ERR_HIP, nmspmm.NM_ERR_UNSUPPORTED)
L = nmspmm.lib()


def no_gpu():
    import torch
    return torch.cuda.device_count() == 0


def weight(n=64, k=100, rows=64, N=8, M=8, **over):
    desc = nmspmm.compress_size(rows, (k + 15) // 16 * 16, N, M)
    w = nmblock.NmScaledWeight(ctypes.pointer(desc), FAKE, FAKE if desc.meta_bytes else None, FAKE, None, n, k)
    for name, value in over.items():
        setattr(w, name, value)
    w.keep = desc
    return w


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(nmblock.NmNorm) == 24
    # 2 pointers, 2 int64, 4 int32, a pointer, a float (padded), 2 norms, 4 pointers
    assert ctypes.sizeof(nmblock.NmNormArgs) == 16 + 16 + 16 + 8 + 8 + 48 + 32
    assert ctypes.sizeof(nmblock.NmNormGradArgs) == 32 + 32 + 16 + 8 + 8 + 48 + 56
    assert ctypes.sizeof(nmblock.NmScaledWeight) == 48
    assert ctypes.sizeof(nmblock.NmGatedGradArgs) == 24 + 8 + 16 + 40


def test_row_codes_refuse():
    f = L.nm_quantize_rows
    assert f(FAKE, 64, 1, -1, 64, FAKE, FAKE, NUL) == SHAPE
    assert f(FAKE, 63, 1, 4, 64, FAKE, FAKE, NUL) == SHAPE           # rows overlap
    assert f(FAKE, 64, 1, 4, 0, FAKE, FAKE, NUL) == SHAPE
    assert f(FAKE, 64, 0, 4, 64, FAKE, FAKE, NUL) == ARG
    assert f(FAKE, 64, 4, 4, 64, FAKE, FAKE, NUL) == ARG
    assert f(NUL, 64, 1, 4, 64, FAKE, FAKE, NUL) == ARG
    assert f(FAKE + 1, 64, 1, 4, 64, FAKE, FAKE, NUL) == ARG         # not aligned to the type
    assert f(FAKE, 64, 1, 4, 64, FAKE + 8, FAKE, NUL) == ARG
    assert f(NUL, 64, 1, 0, 64, NUL, NUL, NUL) == 0                  # no rows


def norm_args(**over):
    one = nmblock.NmNorm(nmblock.NM_NORM_RMS, 1e-6, FAKE, None)
    a = nmblock.NmNormArgs(FAKE, FAKE, 64, 64, 1, 4, 64, 1, None, 1.0, nmblock.NmNorm(), one, FAKE, FAKE, None, None)
    for name, value in over.items():
        setattr(a, name, value)
    return ctypes.byref(a)


def test_norms_refuse():
    f = L.nm_norm_residual
    assert f(NUL, NUL) == ARG
    assert f(norm_args(y=None, r=None), NUL) == ARG
    assert f(norm_args(res=None, z=None), NUL) == ARG
    assert f(norm_args(zq=FAKE), NUL) == ARG                         # codes without scales
    assert f(norm_args(type=5), NUL) == ARG
    assert f(norm_args(m=-1), NUL) == SHAPE
    assert f(norm_args(d=16385, ldy=20000, ldr=20000), NUL) == SHAPE
    assert f(norm_args(groups=3, gate=FAKE), NUL) == SHAPE           # 3 groups of 4 tokens
    assert f(norm_args(groups=2), NUL) == ARG                        # groups of no gate
    assert f(norm_args(ldy=63), NUL) == SHAPE
    assert f(norm_args(pre=nmblock.NmNorm(7, 1e-6, None, None)), NUL) == ARG
    assert f(norm_args(pre=nmblock.NmNorm(1, 0.0, None, None)), NUL) == ARG
    assert f(norm_args(y=FAKE + 1), NUL) == ARG
    assert f(norm_args(m=0, y=None, r=None), NUL) == 0


def grad_args(**over):
    one = nmblock.NmNorm(nmblock.NM_NORM_RMS, 1e-6, FAKE, None)
    a = nmblock.NmNormGradArgs(FAKE, FAKE, FAKE, FAKE, 64, 64, 64, 64, 1, 4, 64, 1, None, 1.0, nmblock.NmNorm(), one,
                               FAKE, FAKE, None, FAKE, None, None, None)
    for name, value in over.items():
        setattr(a, name, value)
    return ctypes.byref(a)


def test_norm_gradients_refuse():
    f, size = L.nm_norm_residual_backward, ctypes.c_size_t()
    assert L.nm_norm_residual_backward_workspace(4, 64, 1, ctypes.byref(size)) == 0 and size.value >= 5 * 64 * 4
    assert L.nm_norm_residual_backward_workspace(0, 64, 1, ctypes.byref(size)) == 0 and size.value == 0
    assert L.nm_norm_residual_backward_workspace(4, 64, 3, ctypes.byref(size)) == SHAPE
    assert L.nm_norm_residual_backward_workspace(4, 64, 1, None) == ARG
    big = 1 << 30
    assert f(NUL, FAKE, big, NUL) == ARG
    assert f(grad_args(), NUL, 0, NUL) == WS
    assert f(grad_args(), FAKE, 16, NUL) == WS
    assert f(grad_args(dz=None, dres=None), FAKE, big, NUL) == ARG
    assert f(grad_args(y=None), FAKE, big, NUL) == ARG               # dy wanted
    assert f(grad_args(res=None), FAKE, big, NUL) == ARG
    assert f(grad_args(dpost_weight=FAKE), FAKE, big, NUL) == ARG    # of a norm that is absent
    assert f(grad_args(lddz=1), FAKE, big, NUL) == SHAPE


def test_products_refuse():
    f, codes = L.nm_linear_i8, L.nm_gemm_i8_scaled
    w, big = weight(), 1 << 30
    ref = ctypes.byref(w)
    assert f(FAKE, 100, 1, -1, ref, FAKE, 64, 1, FAKE, big, NUL) == SHAPE
    assert f(FAKE, 99, 1, 4, ref, FAKE, 64, 1, FAKE, big, NUL) == SHAPE
    assert f(FAKE, 100, 1, 4, ref, FAKE, 63, 1, FAKE, big, NUL) == SHAPE
    assert f(FAKE, 100, 9, 4, ref, FAKE, 64, 1, FAKE, big, NUL) == ARG
    assert f(FAKE, 100, 1, 4, ref, FAKE, 64, 9, FAKE, big, NUL) == ARG
    assert f(NUL, 100, 1, 4, ref, FAKE, 64, 1, FAKE, big, NUL) == ARG
    assert f(FAKE, 100, 1, 400, ref, FAKE, 64, 1, NUL, 0, NUL) == WS
    assert f(FAKE, 100, 1, 400, ref, FAKE, 64, 1, FAKE, 100, NUL) == WS
    assert f(FAKE, 100, 1, 0, ref, NUL, 64, 1, NUL, 0, NUL) == 0
    assert f(FAKE, 100, 1, 4, None, FAKE, 64, 1, FAKE, big, NUL) == ARG
    assert codes(FAKE + 4, FAKE, 4, ref, FAKE, 64, 1, NUL, 0, NUL) == ARG
    assert codes(FAKE, NUL, 4, ref, FAKE, 64, 1, NUL, 0, NUL) == ARG
    short, long = weight(), weight()
    short.k, long.k = 96, 113                                        # the descriptor is of 112 columns
    for bad in (weight(n=65), short, long, weight(n=0), weight(scale=None), weight(scale=FAKE + 4), weight(vals=None)):
        assert codes(FAKE, FAKE, 4, ctypes.byref(bad), FAKE, 200, 1, NUL, 0, NUL) == ARG
    assert codes(FAKE, FAKE, 4, ctypes.byref(weight(k=1 << 17)), FAKE, 64, 1, NUL, 0, NUL) == SHAPE
    size = ctypes.c_size_t()
    assert L.nm_linear_workspace(ref, 400, 1, ctypes.byref(size)) == 0 and size.value >= 400 * 112 + 1600
    assert L.nm_linear_workspace(ref, 400, 0, ctypes.byref(size)) == 0 and size.value == 0
    assert L.nm_linear_workspace(ref, 400, 7, ctypes.byref(size)) == ARG


def test_gated_blocks_refuse():
    g, w = L.nm_gated_i8, weight(n=30, rows=64)                       # 30 channels: 2 x 32 rows
    assert g(FAKE, FAKE, 4, ctypes.byref(w), 0, FAKE, 30, 1, NUL, 0, NUL) == ARG      # no such activation
    assert g(FAKE, FAKE, 4, ctypes.byref(w), 6, FAKE, 30, 1, NUL, 0, NUL) == ARG
    assert g(FAKE, FAKE, 4, ctypes.byref(weight(n=40, rows=64)), 1, FAKE, 40, 1, NUL, 0, NUL) == ARG
    b, size, big = L.nm_gated_backward, ctypes.c_size_t(), 1 << 40
    assert L.nm_gated_backward_workspace(ctypes.byref(w), 100, ctypes.byref(size)) == 0
    assert size.value >= 2 * (100 * 64 + 64 * 128 + 112 * 128 + 112 * 64)
    sparse = weight(n=30, k=96, rows=64, N=2, M=4)
    assert L.nm_gated_backward_workspace(ctypes.byref(sparse), 100, ctypes.byref(size)) == UNSUPPORTED
    assert L.nm_gated_backward_workspace(ctypes.byref(w), 1 << 28, ctypes.byref(size)) == SHAPE

    def args(**over):
        a = nmblock.NmGatedGradArgs(FAKE, FAKE, FAKE, 30, 100, 1, 1, FAKE, FAKE, FAKE, None, None)
        for name, value in over.items():
            setattr(a, name, value)
        return ctypes.byref(a)

    assert b(NUL, ctypes.byref(w), FAKE, big, NUL) == ARG
    assert b(args(type=3), ctypes.byref(w), FAKE, big, NUL) == ARG    # binary32 gradients
    assert b(args(act=9), ctypes.byref(w), FAKE, big, NUL) == ARG
    assert b(args(lddh=29), ctypes.byref(w), FAKE, big, NUL) == SHAPE
    assert b(args(dw_up=None), ctypes.byref(w), FAKE, big, NUL) == ARG
    assert b(args(dh=None), ctypes.byref(w), FAKE, big, NUL) == ARG
    assert b(args(), ctypes.byref(w), FAKE, 100, NUL) == WS
    assert b(args(), ctypes.byref(sparse), FAKE, big, NUL) == UNSUPPORTED


def test_launch_failures_report_nm_err_hip():
    if not no_gpu():
        pytest.skip("a GPU is visible: fake device pointers must not be launched")
    big, w = 1 << 40, weight()
    assert L.nm_quantize_rows(FAKE, 64, 1, 4, 64, FAKE, FAKE, NUL) == HIP
    assert L.nm_norm_residual(norm_args(), NUL) == HIP
    assert L.nm_norm_residual_backward(grad_args(), FAKE, big, NUL) == HIP
    for m in (1, 20, 100, 5000):
        assert L.nm_gemm_i8_scaled(FAKE, FAKE, m, ctypes.byref(w), FAKE, 64, 1, FAKE, big, NUL) == HIP
        assert L.nm_linear_i8(FAKE, 100, 1, m, ctypes.byref(w), FAKE, 64, 1, FAKE, big, NUL) == HIP
    gw = weight(n=30, rows=64)
    a = nmblock.NmGatedGradArgs(FAKE, FAKE, FAKE, 30, 100, 1, 1, FAKE, FAKE, FAKE, None, None)
    assert L.nm_gated_i8(FAKE, FAKE, 4, ctypes.byref(gw), 1, FAKE, 30, 1, NUL, 0, NUL) == HIP
    assert L.nm_gated_backward(ctypes.byref(a), ctypes.byref(gw), FAKE, big, NUL) == HIP


OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump of the ROCm toolchain")
def test_m0_serves_the_loads_to_lds_alone(tmp_path):
    """Every kernel of the built library writes M0 only ahead of a load to LDS (the loads' statements list it as
    clobbered, which the compiler does not promise to honour), and none uses packed binary32 arithmetic."""
    import shutil
    shutil.copy(build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    writes = 0
    for name in os.listdir(tmp_path):
        if not (name.endswith(build.ARCH) and os.path.getsize(tmp_path / name)):
            continue
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp_path, stdout=subprocess.PIPE,
                              text=True) as proc:
            due = 0                                                  # instructions left until the load
            for line in proc.stdout:
                text = line.split("//")[0].strip()
                if not text or text.endswith(":"):
                    continue
                assert not re.match(r"v_pk_(add|mul|fma)_f32", text), text
                if due:
                    due -= 1
                    if "_load_lds_" in text:
                        due = 0
                    else:
                        assert due, f"M0 written, no load to LDS after: {text}"
                if re.search(r"\bm0\b", text):
                    assert re.fullmatch(r"s_mov_b32 m0, s\d+", text), text
                    due, writes = 3, writes + 1
    assert writes > 0


def test_padding_codes_refuses():
    f = L.nm_pad_codes
    assert f(FAKE, 99, 4, 100, FAKE, NUL) == SHAPE
    assert f(FAKE, 100, -1, 100, FAKE, NUL) == SHAPE
    assert f(FAKE, 100, 4, 0, FAKE, NUL) == SHAPE
    assert f(FAKE, 100, 4, 100, FAKE + 8, NUL) == ARG
    assert f(NUL, 100, 4, 100, FAKE, NUL) == ARG
    assert f(NUL, 100, 0, 100, NUL, NUL) == 0
    if no_gpu():
        assert f(FAKE + 1, 101, 4, 100, FAKE, NUL) == HIP


def test_outputs_in_the_memory_of_x_are_not_written_while_it_is_read():
    # few tokens of values go to one kernel that reads x until its end and needs no workspace; where the output shares
    # memory with x the codes are made first, in a workspace
    f, g, lin, gated = L.nm_linear_i8, L.nm_gated, weight(k=64), weight(n=32, k=64)
    x, one = FAKE, NUL
    meets = [(x, 64, 1, 64, 4), (x + 2, 64, 1, 64, 4), (x - 64, 64, 1, 64, 1), (x + 3 * 128 + 126, 64, 1, 64, 4),
             (x, 64, 3, 64, 4), (x + 64, 128, 1, 128, 4), (x + 192, 128, 1, 128, 4), (x, 100, 1, 64, 16)]
    apart = [(x - 512, 64, 1, 64, 4), (x + 4 * 128, 64, 1, 64, 4), (x + 128, 128, 1, 128, 4), (x - 128, 128, 1, 128, 4),
             (x + 128, 64, 1, 64, 1)]
    for out, ldo, otype, ldx, m in meets:
        assert f(x, ldx, 1, m, ctypes.byref(lin), out, ldo, otype, one, 0, NUL) == WS, (out - x, ldo, otype, ldx, m)
        if out % 128 == 0:
            assert g(x, ldx, 1, m, ctypes.byref(gated), 1, out, ldo, otype, one, 0, NUL) == WS
    if no_gpu():       # (the launch fails: the one kernel was chosen)
        for out, ldo, otype, ldx, m in apart:
            assert f(x, ldx, 1, m, ctypes.byref(lin), out, ldo, otype, one, 0, NUL) == HIP, (out - x, ldo, ldx, m)
