"""The entry points of tmamba_seq.h on the host: every declared symbol is
exported and bound, and bad arguments are rejected with the documented status
codes before any launch, in the built library and in a sanitizer build of the
checks.  No test here passes arguments that would reach a kernel launch.  The
binding's refusals are checked on CPU tensors."""

import ctypes
import os
import re
import shutil
import subprocess
import sys

import pytest

from paper_2606_18114_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESHAPE, EALIGN = 1, 2, 3
P = 0x7F0000000000  # a 4 KiB-aligned fake device address, never dereferenced
G = 2 ** 33         # between two fake arrays
BIG = 2 ** 40       # more bytes than any workspace here


@pytest.fixture(scope="module")
def L():
    alt = os.environ.get("TM_ABI_SEQ_LIB")  # the sanitizer build
    if alt:
        lib = ctypes.CDLL(alt)
        for name, (res, args) in ops.SIGNATURES_SEQ.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
        return lib
    if not os.path.exists(ops.lib_path()):
        from paper_2606_18114_amd import build
        build.build(verbose=False)
    return ops.lib()


def test_exports_every_declared_symbol(L):
    text = open(os.path.join(ROOT, "include", "tmamba_seq.h")).read()
    names = set(re.findall(r"^(?:tm_status|int64_t)\s+(tm_[a-z0-9_]+)\(", text, re.M))
    assert names == set(ops.SIGNATURES_SEQ) and len(names) == 13
    for n in names:
        assert hasattr(L, n), n


# the calls with sound arguments, as dicts in the order of the declaration
def _conv():
    return dict(zx=P, f32=0, T=100, nseq=2, H=4, off=P + G, w=P + 2 * G, b=P + 3 * G,
                ring_in=P + 4 * G, pos=P + 5 * G, ring_out=P + 6 * G, u=P + 7 * G, stream=None)


def _conv_bwd():
    return dict(zx=P, f32=0, T=100, nseq=2, H=4, off=P + G, w=P + 2 * G, b=P + 3 * G, du=P + 4 * G,
                dzx=P + 5 * G, dw=P + 6 * G, db=P + 7 * G, ws=P + 8 * G, wsb=BIG, stream=None)


def _scan():
    return dict(u=P, zx=P + G, f32=0, T=1000, nseq=2, H=4, off=P + 2 * G, bias=P + 3 * G,
                alog=P + 4 * G, D=P + 5 * G, s_in=P + 6 * G, s_out=P + 7 * G, y=P + 8 * G,
                ws=P + 9 * G, wsb=BIG, stream=None)


def _scan_bwd():
    return dict(u=P, zx=P + G, f32=0, T=1000, nseq=2, H=4, off=P + 2 * G, bias=P + 3 * G,
                alog=P + 4 * G, D=P + 5 * G, dy=P + 6 * G, dzx=P + 7 * G, du=P + 8 * G,
                dbias=P + 9 * G, dalog=P + 10 * G, dD=P + 11 * G, ws=P + 12 * G, wsb=BIG,
                stream=None)


def _norm():
    return dict(y=P, zx=P + G, f32=0, T=100, nseq=2, H=4, off=P + 4 * G, w=P + 2 * G, eps=1e-5,
                out=P + 3 * G, stream=None)


def _norm_bwd():
    return dict(y=P, zx=P + G, f32=0, T=100, nseq=2, H=4, off=P + 8 * G, w=P + 2 * G, eps=1e-5,
                dout=P + 3 * G, dzx=P + 4 * G, dy=P + 5 * G, dw=P + 6 * G, ws=P + 7 * G, wsb=BIG, stream=None)


def _embed():
    return dict(ids=P, i64=1, T=100, weight=P + G, w_type=0, V=50, D=64, scale=1.0, out=P + 2 * G,
                stream=None)


def _embed_bwd():
    return dict(ids=P, i64=1, T=10000, dout=P + G, V=50, D=64, scale=1.0, dW=P + 2 * G, acc=0,
                ws=P + 3 * G, wsb=BIG, stream=None)


CALLS = {"tm_mixer_conv": _conv, "tm_mixer_conv_bwd": _conv_bwd, "tm_mixer_scan": _scan,
         "tm_mixer_scan_bwd": _scan_bwd, "tm_mixer_norm": _norm, "tm_mixer_norm_bwd": _norm_bwd,
         "tm_embed": _embed, "tm_embed_bwd": _embed_bwd}
OPTIONAL = ("off", "ring_in", "ring_out", "s_in", "s_out", "stream")
POINTERS = ("zx", "off", "w", "b", "ring_in", "pos", "ring_out", "u", "du", "dzx", "dw", "db",
            "ws", "bias", "alog", "D", "s_in", "s_out", "y", "dy", "dbias", "dalog", "dD", "out",
            "dout", "ids", "weight", "dW")
OUTPUTS = ("ring_out", "u_out", "dzx", "dw", "db", "ws", "s_out", "dbias", "dalog", "dD", "out",
           "dW")


def _is_pointer(k, v):
    return k in POINTERS and isinstance(v, int) and v >= P


def call(L, name, **kw):
    args = CALLS[name]()
    assert set(kw) <= set(args), (name, kw)
    args.update(kw)
    return getattr(L, name)(*args.values())


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers(L, name):
    base = CALLS[name]()
    for k, v in base.items():
        if not _is_pointer(k, v):
            continue
        if k not in OPTIONAL:
            assert call(L, name, **{k: 0}) == EINVAL, k
        assert call(L, name, **{k: v + 1}) == EALIGN, k


@pytest.mark.parametrize("name", CALLS)
def test_sizes_and_flags(L, name):
    base = CALLS[name]()
    assert call(L, name, T=0) == ESHAPE
    assert call(L, name, T=2 ** 23 + 1) == ESHAPE
    for k in ("f32", "i64", "acc"):
        if k in base:
            assert call(L, name, **{k: 2}) == EINVAL, k
    if "H" in base:
        assert call(L, name, H=0) == ESHAPE
        assert call(L, name, H=4097) == ESHAPE
    if "nseq" in base:
        assert call(L, name, nseq=0) == ESHAPE
        assert call(L, name, nseq=65536) == ESHAPE
        assert call(L, name, off=0) == EINVAL   # more than one sequence needs offsets
    if "eps" in base:
        for v in (-1.0, float("nan"), float("inf")):
            assert call(L, name, eps=v) == EINVAL
    if "scale" in base:
        for v in (float("nan"), float("inf")):
            assert call(L, name, scale=v) == EINVAL
        for k, most in (("V", 2 ** 23), ("D", 2 ** 30)):
            assert call(L, name, **{k: 0}) == ESHAPE
            assert call(L, name, **{k: most + 1}) == ESHAPE
        assert call(L, name, V=2 ** 23, D=2 ** 30) == ESHAPE  # bytes out of range
    if name == "tm_embed":
        assert call(L, name, w_type=3) == EINVAL
        assert call(L, name, w_type=-1) == EINVAL
    if "wsb" in base:
        assert call(L, name, wsb=0) == ESHAPE
    if name == "tm_mixer_conv":
        assert call(L, name, pos=0) == EINVAL   # a ring needs its position


@pytest.mark.parametrize("name", CALLS)
def test_overlapping_arrays(L, name):
    base = CALLS[name]()
    outs = [k for k in base if _is_pointer(k, base[k])
            and (k in OUTPUTS or (k == "u" and name == "tm_mixer_conv")
                 or (k == "y" and name == "tm_mixer_scan")
                 or (k == "du" and name == "tm_mixer_scan_bwd")
                 or (k == "dy" and name == "tm_mixer_norm_bwd"))]
    assert outs
    for o in outs:
        for k, v in base.items():
            if k == o or not _is_pointer(k, v):
                continue
            if (k, o) in (("ring_in", "ring_out"), ("s_in", "s_out")):
                assert call(L, name, **{o: v + 256}) == EINVAL  # in place is exact or not at all
                continue
            if k in ("ring_out", "s_out") and o in ("ring_in", "s_in"):
                continue
            assert call(L, name, **{o: v}) == EINVAL, (o, k)


def test_workspace_sizes(L):
    assert L.tm_mixer_conv_bwd_workspace(100, 4) > 0
    assert L.tm_mixer_norm_bwd_workspace(100, 4) > 0
    assert L.tm_mixer_scan_workspace(300, 1, 64) == 0
    assert L.tm_mixer_scan_workspace(16384, 1, 64) > 0
    assert L.tm_mixer_scan_bwd_workspace(300, 2, 64) > 0
    assert L.tm_embed_bwd_workspace(10000, 50, 64) > 0
    for f, a in ((L.tm_mixer_conv_bwd_workspace, (0, 4)), (L.tm_mixer_conv_bwd_workspace, (10, 0)),
                 (L.tm_mixer_scan_workspace, (10, 0, 4)), (L.tm_mixer_scan_workspace, (0, 1, 4)),
                 (L.tm_mixer_scan_bwd_workspace, (10, 1, 4097)),
                 (L.tm_mixer_norm_bwd_workspace, (-1, 4)), (L.tm_embed_bwd_workspace, (0, 5, 5)),
                 (L.tm_embed_bwd_workspace, (5, 2 ** 23, 2 ** 30))):
        assert f(*a) == -1, a


def test_segments_of_many_heads(L):
    """The heads fill the chip by themselves: no segments, so no workspace."""
    if os.environ.get("TM_ABI_SEQ_LIB"):
        pytest.skip("sizes of the kernels' own")
    for T, H in ((1000, 512), (1000, 520), (16384, 300), (2 ** 23, 257), (2 ** 20, 4096)):
        assert L.tm_mixer_scan_workspace(T, 1, H) == 0, (T, H)
    assert L.tm_mixer_scan_workspace(16384, 1, 256) > 0


def test_workspaces_of_many_sequences(L):
    """States lie between the segments of a sequence: tokens bound their number,
    not sequences (a state of 64 heads is 2 MiB)."""
    if os.environ.get("TM_ABI_SEQ_LIB"):
        pytest.skip("sizes of the kernels' own")
    T, H, S = 65535, 64, 65535
    assert L.tm_mixer_scan_workspace(T, S, H) == L.tm_mixer_scan_workspace(T, 1, H)
    one, many = L.tm_mixer_scan_bwd_workspace(T, 1, H), L.tm_mixer_scan_bwd_workspace(T, S, H)
    # per sequence and head: six float32 of a chunk's sums
    assert many <= one + 6 * 4 * S * H + 4096
    # one chunk has none: the heads' sums of dB and dC, 1 KiB each, and little else
    assert L.tm_mixer_scan_bwd_workspace(1, 1, H) < 2 ** 17
    assert L.tm_mixer_scan_bwd_workspace(16384, 1024, H) < 2 * 130 * H * 8192 * 4 + 2 ** 28


def test_checks_under_sanitizers(tmp_path):
    if os.environ.get("TM_ABI_SEQ_LIB"):
        pytest.skip("already the sanitizer build")

    def runtime(name):
        out = subprocess.run(["g++", f"-print-file-name={name}"], capture_output=True, text=True)
        path = out.stdout.strip()
        return path if os.path.isabs(path) and os.path.exists(path) else None

    if shutil.which("g++") is None or runtime("libasan.so") is None:
        pytest.skip("g++ with the ASan runtime is needed")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    out = str(tmp_path / "libtmamba_seq_host_asan.so")
    cmd = ["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-Wall", "-Wextra",
           "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
           "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "paper_2606_18114_amd", "csrc", "abi_seq.cpp"),
           os.path.join(ROOT, "tests", "abi_launch_stubs_seq.cpp"),
           "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-o", out]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr
    env = dict(os.environ, LD_PRELOAD=runtime("libasan.so"), TM_ABI_SEQ_LIB=out,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    proc = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                           os.path.abspath(__file__), "-k", "not binding and not modules"],
                          capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    assert proc.returncode == 0, proc.stdout[-3000:] + proc.stderr[-3000:]
    assert "passed" in proc.stdout


def test_binding_refuses_cpu_tensors_and_wrong_types():
    torch = pytest.importorskip("torch")
    bf, f32 = torch.bfloat16, torch.float32
    zx = torch.zeros((5, 2 * 64 + 256 + 1), dtype=bf)
    u, y = torch.zeros((5, 320), dtype=bf), torch.zeros((5, 64), dtype=bf)
    h, c = torch.zeros(1), torch.zeros(320)
    w, nw = torch.zeros((320, 4)), torch.zeros(64)
    for f in (lambda: ops.mixer_conv(zx, w, c), lambda: ops.mixer_conv_bwd(zx, w, c, u, zx),
              lambda: ops.mixer_scan(u, zx, h, h, h),
              lambda: ops.mixer_scan_bwd(u, zx, h, h, h, y, zx),
              lambda: ops.mixer_norm(y, zx, nw), lambda: ops.mixer_norm_bwd(y, zx, nw, y, zx),
              lambda: ops.embed(torch.zeros(3, dtype=torch.int64), torch.zeros((4, 8))),
              lambda: ops.embed_bwd(torch.zeros(3, dtype=torch.int64), torch.zeros((3, 8)), 4)):
        with pytest.raises(ValueError, match="GPU"):
            f()
    with pytest.raises(TypeError):
        ops.mixer_conv([1.0], w, c)
    with pytest.raises(TypeError):
        ops.mixer_conv(zx, w, [1.0])
    with pytest.raises(TypeError):
        ops.mixer_scan(u, zx, h, [1.0], h)
    with pytest.raises(TypeError):
        ops.embed([1], torch.zeros((4, 8), dtype=f32))


def test_modules_refuse_bad_arguments():
    torch = pytest.importorskip("torch")
    from paper_2606_18114_amd.qat import Embedding, Mamba2Mixer
    with pytest.raises(ValueError):
        Mamba2Mixer(0)
    m = Mamba2Mixer(1)
    with pytest.raises(ValueError, match="GPU"):
        m(torch.zeros((4, 385), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        m(torch.zeros((2, 2, 4, 385)))
    with pytest.raises(ValueError):
        m(torch.zeros((2, 4, 385)), offsets=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        Embedding(10, 8)(torch.zeros((2, 3), dtype=torch.int64))
    assert set(m.decode_params()) == {"conv_w", "conv_b", "dt_bias", "A_log", "D", "norm_w"}
