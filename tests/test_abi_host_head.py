"""The entry points of tmamba_head.h on the host: every declared symbol is
exported and bound, and bad arguments are rejected with the documented status
codes before any launch, in the built library and in a sanitizer build of the
checks.  No test here passes arguments that would reach a kernel launch.  The
binding's and the modules' refusals are checked on CPU tensors."""

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
    alt = os.environ.get("TM_ABI_HEAD_LIB")  # the sanitizer build
    if alt:
        lib = ctypes.CDLL(alt)
        for name, (res, args) in ops.SIGNATURES_HEAD.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
        return lib
    if not os.path.exists(ops.lib_path()):
        from paper_2606_18114_amd import build
        build.build(verbose=False)
    return ops.lib()


def test_exports_every_declared_symbol(L):
    text = open(os.path.join(ROOT, "include", "tmamba_head.h")).read()
    names = set(re.findall(r"^(?:tm_status|int64_t)\s+(tm_[a-z0-9_]+)\(", text, re.M))
    assert names == set(ops.SIGNATURES_HEAD) and len(names) == 7
    for n in names:
        assert hasattr(L, n), n


# the calls with sound arguments, as dicts in the order of the declaration
def _loss():
    return dict(h=P, W=P + G, type=1, T=100, V=50, D=64, labels=P + 2 * G, l64=1, ids=P + 3 * G,
                i64=1, top=P + 4 * G, top_type=0, K=5, alpha=0.5, tau=1.0, loss=P + 5 * G,
                stats=P + 6 * G, ws=P + 7 * G, wsb=BIG, stream=None)


def _loss_bwd():
    return dict(h=P, W=P + G, type=2, T=100, V=50, D=64, labels=P + 2 * G, l64=0, ids=P + 3 * G,
                i64=0, K=5, alpha=0.5, tau=2.0, stats=P + 4 * G, dloss=P + 5 * G, dh=P + 6 * G,
                dW=P + 7 * G, dw_type=0, acc=1, ws=P + 8 * G, wsb=BIG, stream=None)


def _norm():
    return dict(r=P, y=P + G, T=100, D=61, w=P + 2 * G, eps=1e-5, r_out=P + 3 * G, x=P + 4 * G,
                stream=None)


def _norm_bwd():
    return dict(r=P, T=100, D=61, w=P + G, eps=1e-5, dx=P + 2 * G, dres=P + 3 * G, dr=P + 4 * G,
                dw=P + 5 * G, ws=P + 6 * G, wsb=BIG, stream=None)


CALLS = {"tm_head_loss": _loss, "tm_head_loss_bwd": _loss_bwd, "tm_block_norm": _norm,
         "tm_block_norm_bwd": _norm_bwd}
OUTPUTS = {"tm_head_loss": ("loss", "stats", "ws"), "tm_head_loss_bwd": ("dh", "dW", "ws"),
           "tm_block_norm": ("r_out", "x"), "tm_block_norm_bwd": ("dr", "dw", "ws")}
# may be null with the rest as it is; may be one array
OPTIONAL = {"tm_block_norm": ("y",), "tm_block_norm_bwd": ("dres",),
            "tm_head_loss_bwd": ("dh", "dW")}
SAME = {("r", "r_out"), ("dres", "dr")}


def _pointers(name):
    return [k for k, v in CALLS[name]().items() if isinstance(v, int) and v >= P]


def call(L, name, **kw):
    args = CALLS[name]()
    assert set(kw) <= set(args), (name, kw)
    args.update(kw)
    return getattr(L, name)(*args.values())


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers(L, name):
    base = CALLS[name]()
    for k in _pointers(name):
        if k not in OPTIONAL.get(name, ()):
            assert call(L, name, **{k: 0}) == EINVAL, k
        assert call(L, name, **{k: base[k] + 1}) == EALIGN, k


@pytest.mark.parametrize("name", CALLS)
def test_overlapping_arrays(L, name):
    base = CALLS[name]()
    for o in OUTPUTS[name]:
        for k in _pointers(name):
            if k == o or (o, k) in SAME:
                continue
            at = base[k] + 256 if (k, o) in SAME else base[k]  # in place is exact or not at all
            assert call(L, name, **{o: at}) == EINVAL, (o, k)


def test_sizes_and_flags_of_the_loss(L):
    for name in ("tm_head_loss", "tm_head_loss_bwd"):
        for k, bad in (("T", (0, -1, 2 ** 23 + 1)), ("V", (0, 2 ** 23 + 1)),
                       ("D", (0, 7, 12, 65544)), ("K", (-1, 1025))):
            for v in bad:
                assert call(L, name, **{k: v}) == ESHAPE, (name, k, v)
        assert call(L, name, T=2 ** 23, K=1024) == ESHAPE
        assert call(L, name, K=0) == EINVAL      # words without a number
        for k, bad in (("type", (0, 3)), ("l64", (2, -1)), ("i64", (2,)),
                       ("alpha", (-0.1, 1.1, float("nan"))),
                       ("tau", (0.0, -1.0, float("nan"), float("inf"), 1e-45, 2.0 ** -11, 2.0 ** 11))):
            for v in bad:
                assert call(L, name, **{k: v}) == EINVAL, (name, k, v)
        assert call(L, name, wsb=0) == ESHAPE
    assert call(L, "tm_head_loss", top_type=3) == EINVAL
    assert call(L, "tm_head_loss", K=0, ids=0) == EINVAL  # logits without words
    assert call(L, "tm_head_loss_bwd", dw_type=1) == EINVAL  # neither float32 nor h's type
    assert call(L, "tm_head_loss_bwd", dw_type=2, acc=1) == EINVAL
    assert call(L, "tm_head_loss_bwd", acc=2) == EINVAL
    assert call(L, "tm_head_loss_bwd", dh=0, dW=0) == EINVAL  # nothing wanted


def test_sizes_of_the_norm(L):
    for name in ("tm_block_norm", "tm_block_norm_bwd"):
        for k, bad in (("T", (0, 2 ** 23 + 1)), ("D", (0, 2 ** 20 + 1))):
            for v in bad:
                assert call(L, name, **{k: v}) == ESHAPE, (name, k, v)
        for v in (-1.0, float("nan"), float("inf")):
            assert call(L, name, eps=v) == EINVAL
    assert call(L, "tm_block_norm_bwd", wsb=0) == ESHAPE
    assert call(L, "tm_block_norm", r_out=0) == EINVAL  # a sum goes somewhere


def test_workspace_sizes(L):
    for f in (L.tm_head_loss_workspace, L.tm_head_loss_bwd_workspace):
        assert f(100, 50, 64) > 0
        for a in ((0, 50, 64), (100, 0, 64), (100, 50, 4), (2 ** 23 + 1, 50, 64)):
            assert f(*a) == -1, a
    assert L.tm_block_norm_bwd_workspace(100, 3) > 0
    assert L.tm_block_norm_bwd_workspace(0, 3) == L.tm_block_norm_bwd_workspace(5, 0) == -1


def test_no_logits_are_kept(L):
    """Forward: the rows and a few sums each.  Backward: a piece of the vocabulary at a time."""
    if os.environ.get("TM_ABI_HEAD_LIB"):
        pytest.skip("sizes of the kernels' own")
    T, V, D = 16384, 50000, 2048
    assert L.tm_head_loss_workspace(T, V, D) < 2 * T * D + 2 ** 23
    assert L.tm_head_loss_bwd_workspace(T, V, D) < 2 ** 29 + 8 * T * D + 2 ** 26
    assert L.tm_head_loss_bwd_workspace(T, 16 * V, D) < 2 ** 29 + 8 * T * D + 2 ** 29
    # many tokens: pieces of 4096 words
    T = 2 ** 20
    assert L.tm_head_loss_bwd_workspace(T, V, 64) < 2 * T * 4096 + 2 * T * 4 * 64 + 2 ** 29


def test_checks_under_sanitizers(tmp_path):
    if os.environ.get("TM_ABI_HEAD_LIB"):
        pytest.skip("already the sanitizer build")

    def runtime(name):
        out = subprocess.run(["g++", f"-print-file-name={name}"], capture_output=True, text=True)
        path = out.stdout.strip()
        return path if os.path.isabs(path) and os.path.exists(path) else None

    if shutil.which("g++") is None or runtime("libasan.so") is None:
        pytest.skip("g++ with the ASan runtime is needed")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    out = str(tmp_path / "libtmamba_head_host_asan.so")
    cmd = ["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-Wall", "-Wextra",
           "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
           "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "paper_2606_18114_amd", "csrc", "abi_head.cpp"),
           os.path.join(ROOT, "tests", "abi_launch_stubs_head.cpp"),
           "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-o", out]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr
    env = dict(os.environ, LD_PRELOAD=runtime("libasan.so"), TM_ABI_HEAD_LIB=out,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    proc = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                           os.path.abspath(__file__), "-k", "not binding and not modules"],
                          capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    assert proc.returncode == 0, proc.stdout[-3000:] + proc.stderr[-3000:]
    assert "passed" in proc.stdout


def test_binding_refuses_cpu_tensors_and_wrong_types():
    torch = pytest.importorskip("torch")
    h, w = torch.zeros((3, 8), dtype=torch.bfloat16), torch.zeros((5, 8), dtype=torch.bfloat16)
    y, f = torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    r, n = torch.zeros((3, 8)), torch.zeros(8)
    for fn in (lambda: ops.head_loss(h, w, y), lambda: ops.head_loss_bwd(h, w, y, f, f),
               lambda: ops.block_norm(r, None, n), lambda: ops.block_norm_bwd(r, n, h)):
        with pytest.raises(ValueError, match="GPU"):
            fn()
    for fn in (lambda: ops.head_loss([1.0], w, y), lambda: ops.head_loss(h, [1.0], y),
               lambda: ops.block_norm([1.0], None, n), lambda: ops.block_norm_bwd([1.0], n, h)):
        with pytest.raises(TypeError):
            fn()


def test_modules_refuse_bad_arguments():
    torch = pytest.importorskip("torch")
    from paper_2606_18114_amd.qat import BlockNorm, Embedding, Head
    head, h = Head(11, 8), torch.zeros((2, 3, 8), dtype=torch.bfloat16)
    y = torch.zeros((2, 3), dtype=torch.int64)
    with pytest.raises(ValueError, match="targets"):
        head(h, torch.zeros(6, dtype=torch.int64))
    with pytest.raises(TypeError, match="bfloat16"):
        head(h.float(), y)
    with pytest.raises(ValueError, match="teacher_logits"):
        head(h, y, y[..., None], torch.zeros((2, 4)))
    with pytest.raises(ValueError, match="GPU"):
        head(h, y)
    emb = Embedding(11, 8)
    assert Head(11, 8, weight=emb.weight).weight is emb.weight
    with pytest.raises(ValueError, match="weight"):
        Head(12, 8, weight=emb.weight)
    norm = BlockNorm(8)
    with pytest.raises(ValueError, match="GPU"):
        norm(torch.zeros((2, 3, 8)))
    with pytest.raises(ValueError, match="residual"):
        norm(torch.zeros((2, 3, 8)), torch.zeros((6, 8)))
