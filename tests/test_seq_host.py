"""Argument checks of the sequence operators (include/mg3m_seq.h), without a
GPU: every refusal comes before anything is launched."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2307_04941_amd import mg3m

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, TOO_LARGE, ALIAS, WORKSPACE, HIP, ALIGN, ARG = 0, 1, 2, 4, 5, 6, 8, 9, 10
P = 1 << 32                                  # addresses that are never read


def at(i):
    return P * (i + 1)


CONV = dict(x=at(0), w=at(1), bias=at(2), state=at(3), y=at(4), begin=0, end=0, ldx=64, ldy=64, T=12, C=64, R=4, N=3,
            load_state=1, silu=1, dtype=1, reserved=0)
SCAN = dict(u=at(0), dt=at(1), A=at(2), B=at(3), C=at(4), D=at(5), z=at(6), dt_bias=at(7), state=at(8), y=at(9),
            begin=0, end=0, workspace=0, workspace_bytes=0, ldu=64, lddt=64, ldb=16, ldc=16, ldz=64, ldy=64, T=12,
            D_=64, G=1, S=16, N=3, load_state=1, softplus=1, dtype=1)
W4 = dict(x=at(0), q=at(1), scale=at(2), zero=at(3), y=at(4), ldx=256, ldy=96, M=4, C=256, K=96, group=64, dtype=1,
          reserved=0)


def call(fn, packer, base, **changes):
    assert set(changes) <= set(base), changes
    a = packer.pack(*{**base, **changes}.values())
    rc = getattr(mg3m.load_library(), fn)(a, None)
    if rc:
        assert mg3m.mg3m_last_error(), rc
    return rc


@pytest.mark.parametrize("fn", ["conv1d_causal_fwd", "conv1d_causal_step", "selective_scan_fwd", "selective_scan_step",
                                "matvec_w4_fwd"])
def test_no_arguments(fn):
    assert getattr(mg3m.load_library(), fn)(None, None) == NULL


def test_argument_structs_match_the_header(tmp_path):
    """The binding packs the structs' bytes itself: sizes and the last field's place as C lays them out."""
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "mg3m_seq.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu\\n", '
                   "sizeof(mg3m_conv1d), offsetof(mg3m_conv1d, T), sizeof(mg3m_scan), offsetof(mg3m_scan, dtype), "
                   "sizeof(mg3m_w4), offsetof(mg3m_w4, M)); return 0; }\n")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", f"-I{ROOT}/include", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    pad = lambda n: -(-n // 8) * 8  # noqa: E731
    assert got == [pad(mg3m._CONV1D.size), 72, pad(mg3m._SCAN.size), mg3m._SCAN.size - 4, pad(mg3m._W4.size), 56]


@pytest.mark.parametrize("change,rc", [
    (dict(x=0), NULL), (dict(w=0), NULL), (dict(y=0), NULL), (dict(state=0), NULL),
    (dict(x=P + 1), ALIGN), (dict(state=at(3) + 1), ALIGN), (dict(y=at(4) + 2, dtype=0), ALIGN),
    (dict(begin=at(5) + 2, end=at(6)), ALIGN),
    (dict(C=0), SHAPE), (dict(R=0), SHAPE), (dict(R=9), SHAPE), (dict(N=0), SHAPE), (dict(T=-1), SHAPE),
    (dict(T=13), SHAPE), (dict(ldx=63), SHAPE), (dict(ldy=(1 << 30) + 1), SHAPE),
    (dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(silu=2), ARG), (dict(load_state=-1), ARG), (dict(reserved=1), ARG),
    (dict(begin=at(5)), ARG), (dict(end=at(5)), ARG),
    (dict(y=at(0)), ALIAS), (dict(y=at(0) + 2), ALIAS), (dict(y=at(3)), ALIAS), (dict(state=at(0)), ALIAS),
    (dict(y=at(1) + 64), ALIAS), (dict(bias=at(4)), ALIAS), (dict(begin=at(4), end=at(5)), ALIAS),
    (dict(x=at(4) + 64, ldx=128, ldy=128), ALIAS)])
def test_conv_refusals(change, rc):
    assert call("conv1d_causal_fwd", mg3m._CONV1D, CONV, **change) == rc


@pytest.mark.parametrize("change,rc", [
    (dict(state=0), NULL), (dict(x=0), NULL), (dict(begin=at(5), end=at(6)), ARG), (dict(N=0), SHAPE),
    (dict(y=at(0)), ALIAS), (dict(R=9), SHAPE), (dict(dtype=7), ARG)])
def test_conv_step_refusals(change, rc):
    assert call("conv1d_causal_step", mg3m._CONV1D, CONV, **change) == rc


@pytest.mark.parametrize("change,rc", [
    (dict(u=0), NULL), (dict(dt=0), NULL), (dict(A=0), NULL), (dict(B=0), NULL), (dict(C=0), NULL), (dict(y=0), NULL),
    (dict(state=0), NULL), (dict(u=P + 1), ALIGN), (dict(A=at(2) + 2), ALIGN), (dict(state=at(8) + 2), ALIGN),
    (dict(D_=0), SHAPE), (dict(G=0), SHAPE), (dict(G=3), SHAPE), (dict(S=0), SHAPE), (dict(S=257), SHAPE),
    (dict(N=0), SHAPE), (dict(T=-3), SHAPE), (dict(T=14), SHAPE), (dict(ldb=15), SHAPE), (dict(ldz=1), SHAPE),
    (dict(D_=1 << 24, S=256, ldu=1 << 24, lddt=1 << 24, ldz=1 << 24, ldy=1 << 24, ldb=256, ldc=256), TOO_LARGE),
    (dict(dtype=3), ARG), (dict(softplus=2), ARG), (dict(load_state=3), ARG), (dict(end=at(9)), ARG),
    (dict(y=at(0)), ALIAS), (dict(y=at(6)), ALIAS), (dict(state=at(2)), ALIAS), (dict(dt_bias=at(9)), ALIAS),
    (dict(y=at(3) + 8), ALIAS), (dict(y=at(8)), ALIAS)])
def test_scan_refusals(change, rc):
    assert call("selective_scan_fwd", mg3m._SCAN, SCAN, **change) == rc


@pytest.mark.parametrize("change,rc", [(dict(state=0), NULL), (dict(begin=at(12), end=at(13)), ARG), (dict(S=300), SHAPE),
                                       (dict(y=at(0)), ALIAS), (dict(state=at(8) + 1), ALIGN)])
def test_scan_step_refusals(change, rc):
    assert call("selective_scan_step", mg3m._SCAN, SCAN, **change) == rc


def test_scan_workspace():
    lib = mg3m.load_library()
    b = ctypes.c_size_t()
    assert lib.selective_scan_workspace_bytes(12, 64, 1, 16, 3, None) == NULL
    for bad in ((-1, 64, 1, 16, 3), (12, 0, 1, 16, 3), (12, 64, 3, 16, 3), (12, 64, 1, 0, 3), (12, 64, 1, 16, 0)):
        assert lib.selective_scan_workspace_bytes(*bad, ctypes.byref(b)) == SHAPE
    need = mg3m.selective_scan_workspace_bytes(4096, 512, 1, 16, 1)
    assert need < 4096 * 512 * 16 * 4 / 8                       # far below one state per token
    big = dict(T=4096, D_=512, N=1, ldu=512, lddt=512, ldz=512, ldy=512)
    if need:
        assert call("selective_scan_fwd", mg3m._SCAN, SCAN, **big, workspace=at(20), workspace_bytes=need - 1) == WORKSPACE
        assert call("selective_scan_fwd", mg3m._SCAN, SCAN, **big, workspace=at(20) + 8, workspace_bytes=need) == WORKSPACE
        assert call("selective_scan_fwd", mg3m._SCAN, SCAN, **big, workspace=at(0), workspace_bytes=need) == ALIAS


@pytest.mark.parametrize("change,rc", [
    (dict(x=0), NULL), (dict(q=0), NULL), (dict(scale=0), NULL), (dict(y=0), NULL),
    (dict(q=at(1) + 8), ALIGN), (dict(x=P + 1), ALIGN), (dict(scale=at(2) + 1), ALIGN),
    (dict(M=0), SHAPE), (dict(C=0), SHAPE), (dict(K=0), SHAPE), (dict(group=16), SHAPE), (dict(group=48), SHAPE),
    (dict(group=96), SHAPE), (dict(group=0), SHAPE), (dict(ldx=255), SHAPE), (dict(ldy=95), SHAPE),
    (dict(dtype=3), ARG), (dict(reserved=2), ARG),
    (dict(y=at(0)), ALIAS), (dict(y=at(1) + 32), ALIAS), (dict(y=at(2)), ALIAS), (dict(y=at(3)), ALIAS)])
def test_w4_refusals(change, rc):
    assert call("matvec_w4_fwd", mg3m._W4, W4, **change) == rc


def test_columns_of_one_tensor_are_no_alias():
    """Outputs between the inputs' rows pass the checks: without a GPU the
    call then fails at its launch, with one it is not made here."""
    if torch.cuda.is_available():
        pytest.skip("addresses are made up")
    assert call("conv1d_causal_fwd", mg3m._CONV1D, CONV, x=at(0), y=at(0) + 128, ldx=192, ldy=192) == HIP
    assert call("conv1d_causal_fwd", mg3m._CONV1D, CONV, x=at(0), y=at(0) + 126, ldx=192, ldy=192) == ALIAS
    assert call("conv1d_causal_fwd", mg3m._CONV1D, CONV, x=at(0), y=at(0) + 258, ldx=192, ldy=192) == ALIAS


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        mg3m.conv1d_causal(x, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="GPU"):
        mg3m.conv1d_causal_step(x, torch.zeros(4, 8), torch.zeros(4, 3, 8))
    with pytest.raises(ValueError, match="GPU"):
        mg3m.selective_scan(x, x, torch.zeros(8, 2), torch.zeros(4, 2), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="GPU"):
        mg3m.matvec_w4(x, torch.zeros(3, 4, dtype=torch.uint8), torch.zeros(3, 1))


class Row:
    """Enough of a tensor for the binding's row checks."""

    def __init__(self, shape, strides):
        self.shape, self._s = shape, strides

    def stride(self):
        return self._s


@pytest.mark.parametrize("shape,strides,tail,ld", [
    ((5, 8), (20, 1), 1, 20), ((2, 5, 8), (100, 20, 1), 1, 20), ((1, 5, 8), (7, 20, 1), 1, 20), ((6, 1, 8), (20, 3, 1), 1, 20),
    ((1, 8), (999, 1), 1, 8), ((4, 2, 8), (50, 8, 1), 2, 50), ((4, 1, 8), (50, 99, 1), 2, 50), ((4, 1), (50, 7), 1, 50),
    ((2, 5, 8), (101, 20, 1), 1, None), ((5, 8), (20, 2), 1, None), ((4, 2, 8), (50, 9, 1), 2, None)])
def test_row_distances(shape, strides, tail, ld):
    if ld is None:
        with pytest.raises(ValueError):
            mg3m._row_distance(Row(shape, strides), "x", tail)
    else:
        assert mg3m._row_distance(Row(shape, strides), "x", tail) == ld


def test_every_entry_point_is_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mg3m_seq.h")).read(), flags=re.S)
    names = re.findall(r"^int (\w+)\(", text, flags=re.M)
    assert len(names) == 6
    for n in names:
        assert getattr(mg3m.load_library(), n).argtypes is not None, n


def test_pieces_of_sequences(tmp_path):
    """tests/seq_pieces.cpp under the address and undefined-behaviour sanitizers."""
    exe = tmp_path / "pieces"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{ROOT}/paper_2307_04941_amd/csrc", os.path.join(ROOT, "tests", "seq_pieces.cpp"), "-o", str(exe)],
                   check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "pieces ok" in run.stdout, run.stdout + run.stderr


@pytest.mark.parametrize("fn,packer,base,change", [
    ("conv1d_causal_fwd", "_CONV1D", "CONV", dict(T=0x7fff0001, N=1)),
    ("conv1d_causal_fwd", "_CONV1D", "CONV", dict(C=(1 << 30) + 1, ldx=1 << 30, ldy=1 << 30)),
    ("selective_scan_fwd", "_SCAN", "SCAN", dict(T=0x7fff0001, N=1)),
    ("selective_scan_fwd", "_SCAN", "SCAN", dict(D_=(1 << 26) + 64, ldu=1 << 27, lddt=1 << 27, ldz=1 << 27, ldy=1 << 27)),
    ("matvec_w4_fwd", "_W4", "W4", dict(K=(1 << 30) + 1, ldy=1 << 30)),
    ("matvec_w4_fwd", "_W4", "W4", dict(M=(1 << 30) + 1)),
    ("matvec_w4_fwd", "_W4", "W4", dict(C=(1 << 20) + 64, ldx=1 << 21))])
def test_sizes_past_the_kernels_counters(fn, packer, base, change):
    assert call(fn, getattr(mg3m, packer), globals()[base], **change) == TOO_LARGE


@pytest.mark.parametrize("fn,packer,base", [("conv1d_causal_fwd", "_CONV1D", CONV), ("conv1d_causal_step", "_CONV1D", CONV),
                                            ("selective_scan_fwd", "_SCAN", SCAN), ("selective_scan_step", "_SCAN", SCAN),
                                            ("matvec_w4_fwd", "_W4", W4)])
def test_injected_launch_failure(fn, packer, base, monkeypatch):
    """Valid arguments pass every check and reach the launch, which fails."""
    monkeypatch.setenv("MG3M_TEST_FAIL_LAUNCH", "1")
    assert call(fn, getattr(mg3m, packer), base) == HIP
    assert "MG3M_TEST_FAIL_LAUNCH" in mg3m.mg3m_last_error()


def test_more_threads_than_a_launch_takes():
    """Grids are counted in threads of 32 bits: 2^33 are refused."""
    far = dict(state=at(1000), ldb=16, ldc=16)
    assert call("selective_scan_step", mg3m._SCAN, SCAN, N=1 << 11, D_=1 << 20, ldu=1 << 20, lddt=1 << 20, ldz=1 << 20,
                ldy=1 << 20, **far) == TOO_LARGE
    assert call("selective_scan_fwd", mg3m._SCAN, SCAN, T=1 << 20, N=1 << 20, D_=1024, ldu=1024, lddt=1024, ldz=1024,
                ldy=1024, state=0, load_state=0) == TOO_LARGE
    assert call("matvec_w4_fwd", mg3m._W4, W4, M=1 << 16, K=1 << 18, ldy=1 << 18, C=32, group=32, ldx=32,
                y=at(1000)) == TOO_LARGE


def test_quick_binding_leaves_the_rest_to_python():
    """_seq_torch takes ordinary GPU tensors only: for anything else it does nothing and returns None."""
    quick = mg3m.load_binding()
    x = torch.zeros(4, 8)
    assert quick.conv1d(False, x, x, None, True, None, False, None, None, None, None) is None
    assert quick.conv1d(False, None, x, None, True, None, False, None, None, None, None) is None
    assert quick.conv1d(False, x) is None and quick.w4() is None
    assert quick.scan(True, x, x, x, x, x, None, None, None, True, x, True, None, None, None, None) is None
    assert quick.w4(x, torch.zeros(3, 4, dtype=torch.uint8), x, None, None) is None
    with pytest.raises(ValueError):
        quick.bind(1, 2)
