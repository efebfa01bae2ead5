"""Host side of rotary positions and differential attention (CPU): argument checks that come before any launch, workspaces,
struct layouts, the binding's refusals, and the compiled kernels' loads to LDS."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_12505_amd import build, nmattention as na, nmspmm

FAKE, NUL = 1 << 20, None
OK, ARG, SHAPE, WS = nmspmm.NM_OK, nmspmm.NM_ERR_ARG, nmspmm.NM_ERR_SHAPE, nmspmm.NM_ERR_WORKSPACE
L = nmspmm.lib()


def test_struct_sizes_match_the_header(tmp_path):
    names = dict(nm_rotary_part=na.NmRotaryPart, nm_rotary_args=na.NmRotaryArgs, nm_heads=na.NmHeads, nm_tokens=na.NmTokens,
                 nm_diff_weight=na.NmDiffWeight, nm_diff_args=na.NmDiffArgs, nm_diff_grad_args=na.NmDiffGradArgs)
    lines = []
    for c, p in names.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f} %zu\\n", offsetof({c}, {f}));' for f, _ in p._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "nmspmm.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", f"-I{build.INCLUDE}", str(src), "-o", str(tmp_path / "sizes")], check=True)
    out = dict(l.rsplit(" ", 1) for l in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True,
                                                       check=True).stdout.splitlines())
    for c, p in names.items():
        assert int(out[c]) == ctypes.sizeof(p), c
        for f, _ in p._fields_:
            assert int(out[f"{c}.{f}"]) == getattr(p, f).offset, (c, f)


@pytest.mark.parametrize("structure", [na.NmRotaryArgs, na.NmDiffArgs, na.NmDiffGradArgs])
def test_packed_values_are_the_structure(structure):
    pack = na._packer(structure)
    assert pack.size == ctypes.sizeof(structure)
    count = len(pack.unpack(bytes(pack.size)))
    raw = pack.pack(*range(1, count + 1))
    s = structure.from_buffer_copy(raw)
    seen = []

    def walk(v):
        if isinstance(v, ctypes.Structure):
            for f, _ in v._fields_:
                walk(getattr(v, f))
        elif isinstance(v, ctypes.Array):
            for x in v:
                walk(x)
        else:
            seen.append(int(v))
    walk(s)
    assert seen == list(range(1, count + 1))


def rotary(**over):
    a = na.NmRotaryArgs()
    a.part[0] = na.NmRotaryPart(FAKE, FAKE, 64, 32, 64, 32, 2)
    a.pos, a.ld_pos, a.freq, a.axis, a.tokens = FAKE, 4, FAKE, FAKE, 4
    a.type, a.pairs, a.d, a.axes = 1, 8, 32, 2
    for name, value in over.items():
        if name.startswith("p_"):
            setattr(a.part[0], name[2:], value)
        else:
            setattr(a, name, value)
    return ctypes.byref(a)


def test_rotary_refuses():
    f = L.nm_rotary
    assert f(NUL, NUL) == ARG
    for bad in (dict(type=0), dict(type=4), dict(p_x=None), dict(p_out=None), dict(p_x=FAKE + 1), dict(pos=None), dict(freq=None),
                dict(axis=None), dict(pos=FAKE + 2), dict(freq=FAKE + 4), dict(p_heads=0)):
        assert f(rotary(**bad), NUL) == ARG, bad
    for bad in (dict(tokens=-1), dict(pairs=0), dict(pairs=17), dict(d=1025), dict(axes=0), dict(ld_pos=-1), dict(p_heads=-1),
                dict(p_x_token=-1), dict(p_out_head=-1), dict(p_heads=1 << 16)):
        assert f(rotary(**bad), NUL) == SHAPE, bad
    assert f(rotary(tokens=0, p_x=None, pos=None), NUL) == OK


def heads(token=128, head=32, batch=1 << 14, p=FAKE):
    return na.NmHeads(p, batch, token, head)


def diff(**over):
    a = na.NmDiffArgs()
    a.q, a.k, a.v, a.o = heads(), heads(), heads(), heads()
    a.tokens = na.NmTokens(2, 100, 100, -1, 0, None, None, None, None, 0, 0)
    a.weight = na.NmDiffWeight(FAKE)
    a.type, a.H, a.Hk, a.d, a.dv, a.scale = 1, 2, 2, 32, 64, 0.1
    return change(a, over)


def change(a, over):
    for name, value in over.items():
        at = a
        *path, last = name.split("__")
        for p in path:
            at = getattr(at, p)
        setattr(at, last, value)
    return a


BAD_ARG = [dict(type=3), dict(type=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
           dict(q__p=None), dict(k__p=None), dict(v__p=FAKE + 1), dict(weight__value=FAKE + 2),
           dict(tokens__q_offsets=FAKE), dict(tokens__q_lens=FAKE + 1),
           dict(tokens__q_offsets=FAKE, tokens__k_offsets=FAKE, tokens__k_lens=FAKE),
           dict(weight__value=None, weight__n=4)]
BAD_SHAPE = [dict(H=0), dict(Hk=0), dict(H=3), dict(d=0), dict(d=129), dict(H=1 << 16, Hk=1), dict(tokens__batch=-1),
             dict(tokens__tq=-1), dict(tokens__tk=1 << 28), dict(k__token=-1), dict(v__token=1 << 22), dict(q__head=-1),
             dict(weight__value=None, weight__n=0), dict(tokens__q_offsets=FAKE, tokens__k_offsets=FAKE, tokens__total_q=-1)]


def test_attention_refuses():
    f, size = L.nm_diff_attention, ctypes.c_size_t()
    assert f(NUL, NUL, 0, NUL) == ARG and L.nm_diff_attention_workspace(NUL, ctypes.byref(size)) == ARG
    assert L.nm_diff_attention_workspace(ctypes.byref(diff()), None) == ARG
    for bad in BAD_ARG + [dict(o__p=None), dict(o__p=FAKE + 1), dict(kept=FAKE), dict(stats=FAKE), dict(kept=FAKE + 2, stats=FAKE)]:
        assert f(ctypes.byref(diff(**bad)), FAKE, 1 << 40, NUL) == ARG, bad
    for bad in BAD_SHAPE + [dict(dv=257), dict(dv=0)]:
        assert f(ctypes.byref(diff(**bad)), FAKE, 1 << 40, NUL) == SHAPE, bad
    assert f(ctypes.byref(diff(tokens__batch=1 << 23, tokens__tq=1, tokens__tk=1)), NUL, 0, NUL) == SHAPE   # a launch's size
    for nothing in (dict(tokens__batch=0), dict(tokens__tq=0, q__p=None, o__p=None)):
        assert f(ctypes.byref(diff(**nothing)), NUL, 0, NUL) == OK
    # few rows over long keys need a workspace for their parts
    long = diff(tokens__tq=1, tokens__tk=100000)
    assert L.nm_diff_attention_workspace(ctypes.byref(long), ctypes.byref(size)) == OK
    assert size.value >= 2 * 2 * 2 * (2 * 64 + 4) * 4
    assert f(ctypes.byref(long), NUL, 0, NUL) == WS and f(ctypes.byref(long), FAKE, size.value - 1, NUL) == WS
    assert f(ctypes.byref(long), FAKE + 8, size.value, NUL) == WS
    assert L.nm_diff_attention_workspace(ctypes.byref(diff()), ctypes.byref(size)) == OK and size.value == 0


def grad(**over):
    a = na.NmDiffGradArgs()
    a.q, a.k, a.v, a.grad_o, a.dq, a.dk, a.dv = (heads() for _ in range(7))
    a.kept, a.stats, a.dlam = FAKE, FAKE, FAKE
    a.tokens = na.NmTokens(2, 100, 100, -1, 0, None, None, None, None, 0, 0)
    a.weight = na.NmDiffWeight(FAKE)
    a.type, a.H, a.Hk, a.d, a.dv_width, a.scale = 1, 2, 2, 32, 64, 0.1
    return change(a, over)


def test_gradients_refuse():
    f, size = L.nm_diff_attention_backward, ctypes.c_size_t()
    assert f(NUL, FAKE, 1 << 40, NUL) == ARG
    for bad in BAD_ARG + [dict(grad_o__p=None), dict(dq__p=None), dict(dk__p=None), dict(dv__p=FAKE + 1), dict(kept=None),
                          dict(stats=None), dict(dlam=None), dict(dlam=FAKE + 2),
                          dict(weight__value=None, weight__q1=FAKE, weight__k1=FAKE, weight__q2=FAKE, weight__k2=FAKE,
                               weight__n=4)]:
        assert f(ctypes.byref(grad(**bad)), FAKE, 1 << 40, NUL) == ARG, bad
    for bad in BAD_SHAPE + [dict(dv_width=257)]:
        assert f(ctypes.byref(grad(**bad)), FAKE, 1 << 40, NUL) == SHAPE, bad
    assert L.nm_diff_attention_backward_workspace(ctypes.byref(grad()), ctypes.byref(size)) == OK
    assert size.value >= 2 * 2 * 200 * 4 + 2 * 2 * 16
    assert f(ctypes.byref(grad()), NUL, 0, NUL) == WS and f(ctypes.byref(grad()), FAKE, size.value - 1, NUL) == WS
    # the tensors' 2^32 values of work: sizes in 64 bits
    big = grad(tokens__batch=1 << 10, tokens__tq=1 << 20, H=64, Hk=64)
    assert L.nm_diff_attention_backward_workspace(ctypes.byref(big), ctypes.byref(size)) == OK
    assert size.value > 2 * 64 * (1 << 30) * 4


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(3, 2, 16)
    with pytest.raises(ValueError):
        na.rotary(x, torch.zeros(1, 3, dtype=torch.int32), na.RotaryAxes([1.0], [0], device="cpu"))
    with pytest.raises(ValueError):
        na.DiffWeight(torch.zeros(2))
    for bad in (dict(style="thirds"), dict(freqs=[]), dict(axis=[0, 1]), dict(axis=[-1])):
        with pytest.raises(ValueError):
            na.RotaryAxes(**{**dict(freqs=[1.0], axis=[0], device="cpu"), **bad})
    axes = na.RotaryAxes.of_sections((2, 1), theta=100.0, device="cpu")
    assert axes.axis.tolist() == [0, 0, 1] and axes.axes == 2 and axes.pairs == 3
    assert axes.freqs.tolist() == [1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3)]
    own = na.RotaryAxes.of_sections((2, 2), theta=100.0, own_ladders=True, device="cpu")
    assert own.freqs.tolist() == [1.0, 0.1, 1.0, 0.1]


HIPCC = shutil.which("hipcc") or ("/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else None)


@pytest.mark.skipif(HIPCC is None, reason="hipcc not available")
@pytest.mark.parametrize("name", ["nmspmm_attn.hip", "nmspmm_attn_grad.hip"])
def test_loads_to_lds_have_m0_and_their_wait_states(tmp_path, name):
    """M0 is written for loads to LDS alone, each write with its wait states before its load: five after a vector
    instruction's write of a scalar register that the load reads."""
    out = tmp_path / "kernels.s"
    subprocess.run([HIPCC, *build.FLAGS, "--cuda-device-only", "-S", f"-I{build.INCLUDE}", os.path.join(build.CSRC, name), "-o",
                    str(out)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL, timeout=600)
    lines = []
    for raw in out.read_text().splitlines():
        s = raw.split(";")[0].strip()
        if s and not s.startswith(".") and not s.endswith(":"):
            lines.append(s)
    writes = 0
    for i, s in enumerate(lines):
        if "_load_lds_" in s:
            assert re.search(r"\bm0\b", lines[i - 2]) and lines[i - 1] == "s_nop 4", s
        if not re.search(r"\bm0\b", s):
            continue
        assert re.fullmatch(r"s_mov_b32 m0, s\d+", s), s
        assert lines[i + 1] == "s_nop 4" and "_load_lds_dword" in lines[i + 2], (s, lines[i + 1], lines[i + 2])
        writes += 1
    assert writes > 0
