"""C-ABI and wrapper checks, without a GPU, of the operators around the layer: block-scaled formats
and their expert MLP, the norm and its backward, the few-token layer.  Every call below fails
validation or has nothing to do, so no pointer is dereferenced."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2607_18631_amd import moe
from paper_2607_18631_amd import workloads as wl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_18631_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "host_sanitizer")

FAKE = ctypes.c_void_p(0x100000)        # aligned, never dereferenced
OFF8 = ctypes.c_void_p(0x100008)
OFF2 = ctypes.c_void_p(0x100002)
BIG = 1 << 44

INVALID, UNSUPPORTED, WORKSPACE = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED, moe.MOE_ERR_WORKSPACE
BASE = wl.MoEShape(T=8, d=64, E=8, top_k=2, F=96, E_local=8)


def status(fn, *args):
    st = fn(*args)
    return st, moe.last_error()


def refused(result, st, needle):
    assert result[0] == st and needle in result[1], result


# ---- block-scaled conversion ----
def convert(rows=4, cols=64, fmt=moe.MOE_MX_E4M3, x=FAKE, q=FAKE, s=FAKE, back=False):
    L = moe.lib()
    return status(L.moe_mx_dequantize, rows, cols, fmt, q, s, x, None) if back else \
        status(L.moe_mx_quantize, rows, cols, fmt, x, q, s, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,st,needle", [
    (dict(rows=-1), INVALID, "rows (-1) < 0"),
    (dict(cols=0), INVALID, "cols (0) <= 0"),
    (dict(cols=-32), INVALID, "cols (-32) <= 0"),
    (dict(cols=48), UNSUPPORTED, "cols (48) % 32 != 0"),
    (dict(rows=1 << 35, cols=32), UNSUPPORTED, "2^40"),
    (dict(fmt=2), UNSUPPORTED, "format (2)"),
    (dict(fmt=-1), UNSUPPORTED, "format (-1)"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(q=None), INVALID, "elements is NULL"),
    (dict(s=None), INVALID, "scales is NULL"),
    (dict(x=OFF8), INVALID, "x"),
    (dict(q=OFF8), INVALID, "elements"),
    (dict(s=OFF8), INVALID, "scales"),
])
def test_conversion_refusals(back, kw, st, needle):
    refused(convert(back=back, **kw), st, needle)


@pytest.mark.parametrize("back", [False, True])
def test_conversion_of_no_rows(back):
    assert convert(rows=0, x=None, q=None, s=None, back=back) == (moe.MOE_OK, "")


# ---- norm ----
def norm(rows=4, d=64, eps=1e-6, x=FAKE, residual=FAKE, gamma=FAKE, h=FAKE, y=FAKE, q=FAKE, s=FAKE, rstd=FAKE):
    return status(moe.lib().moe_add_rmsnorm, rows, d, eps, x, residual, gamma, h, y, q, s, rstd, None)


@pytest.mark.parametrize("kw,st,needle", [
    (dict(rows=-1), INVALID, "rows (-1) < 0"),
    (dict(rows=1 << 31), UNSUPPORTED, "2^31"),
    (dict(d=0), INVALID, "d (0) <= 0"),
    (dict(d=12, q=None, s=None), UNSUPPORTED, "d (12) % 8 != 0"),
    (dict(d=40), UNSUPPORTED, "d (40) % 32 != 0"),
    (dict(eps=-1.0), INVALID, "eps"),
    (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"),
    (dict(x=None), INVALID, "x is NULL"),
    (dict(gamma=None), INVALID, "gamma is NULL"),
    (dict(h=None), INVALID, "h is NULL"),
    (dict(residual=None), INVALID, "h is given without a residual"),
    (dict(y=None, q=None, s=None), INVALID, "y and y_q are both NULL"),
    (dict(q=None), INVALID, "y_q is NULL"),
    (dict(s=None), INVALID, "y_scales is NULL"),
    (dict(x=OFF8), INVALID, "x"),
    (dict(residual=OFF8), INVALID, "residual"),
    (dict(h=OFF8), INVALID, "h"),
    (dict(y=OFF8), INVALID, "y"),
    (dict(q=OFF8), INVALID, "y_q"),
    (dict(s=OFF8), INVALID, "y_scales"),
    (dict(rstd=OFF2), INVALID, "rstd"),
])
def test_norm_refusals(kw, st, needle):
    refused(norm(**kw), st, needle)


def test_norm_of_no_rows():
    assert norm(rows=0, x=None, residual=None, gamma=None, h=None, y=None, q=None, s=None, rstd=None) == (moe.MOE_OK, "")


def norm_bwd(rows=4, d=64, dy=FAKE, dh=FAKE, h=FAKE, gamma=FAKE, rstd=FAKE, dx=FAKE, dg=FAKE, ws=FAKE, ws_bytes=BIG):
    return status(moe.lib().moe_add_rmsnorm_backward, rows, d, dy, dh, h, gamma, rstd, dx, dg, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,st,needle", [
    (dict(rows=-1), INVALID, "rows (-1) < 0"),
    (dict(d=-8), INVALID, "d (-8) <= 0"),
    (dict(d=12), UNSUPPORTED, "d (12) % 8 != 0"),
    (dict(dy=None), INVALID, "dy is NULL"),
    (dict(h=None), INVALID, "h is NULL"),
    (dict(gamma=None), INVALID, "gamma is NULL"),
    (dict(rstd=None), INVALID, "rstd is NULL"),
    (dict(dx=None), INVALID, "dx is NULL"),
    (dict(dg=None), INVALID, "dgamma is NULL"),
    (dict(rows=0, dg=None), INVALID, "dgamma is NULL"),
    (dict(dh=OFF8), INVALID, "dh"),
    (dict(ws=None), WORKSPACE, "workspace is NULL"),
    (dict(ws_bytes=16), WORKSPACE, "required"),
])
def test_norm_backward_refusals(kw, st, needle):
    refused(norm_bwd(**kw), st, needle)


def test_norm_workspace():
    for rows, d in ((0, 8), (1, 8), (4096, 7168), ((1 << 31) - 1, 16384)):
        n = moe.add_rmsnorm_workspace_size(rows, d)
        assert n % 256 == 0 and d * 4 <= n <= 1 << 32
    for rows, d, needle in ((-1, 8, "rows"), (1, 0, "d (0)"), (1, 12, "d (12)")):
        with pytest.raises(moe.MoEError, match="rows|d "):
            moe.add_rmsnorm_workspace_size(rows, d)
        assert needle in moe.last_error()


# ---- expert MLP ----
def mlp(sh, fmt=moe.MOE_MX_E4M3, ws=FAKE, ws_bytes=BIG, **ptr):
    names = ("x_q", "x_scales", "offsets", "w13_q", "w13_scales", "w2_q", "w2_scales", "y_perm")
    shape = None if sh is None else ctypes.byref(moe.shape_c(sh))
    return status(moe.lib().moe_mx_grouped_ffn, shape, fmt, *(ptr.get(n, FAKE) for n in names), ws, ws_bytes, None)


@pytest.mark.parametrize("change,kw,st,needle", [
    (dict(d=72), {}, UNSUPPORTED, "d (72) % 32 != 0"),
    (dict(F=40), {}, UNSUPPORTED, "F (40) % 32 != 0"),
    (dict(d=1 << 16, F=1 << 15), {}, UNSUPPORTED, "d * F"),
    (dict(d=1 << 20, F=32), {}, UNSUPPORTED, "d or F (1048576) >= 2^20"),
    (dict(d=32, F=1 << 20), {}, UNSUPPORTED, "d or F (1048576) >= 2^20"),
    (dict(top_k=9), {}, UNSUPPORTED, "top_k (9)"),
    ({}, dict(fmt=2), UNSUPPORTED, "format (2)"),
    ({}, dict(ws=None), WORKSPACE, "workspace is NULL"),
    ({}, dict(ws_bytes=255), WORKSPACE, "required"),
])
def test_mlp_refusals(change, kw, st, needle):
    refused(mlp(BASE.replace(**change), **kw), st, needle)


@pytest.mark.parametrize("name", ["x_q", "x_scales", "offsets", "w13_q", "w13_scales", "w2_q", "w2_scales", "y_perm"])
def test_mlp_pointers(name):
    refused(mlp(BASE, **{name: None}), INVALID, f"{name} is NULL")
    refused(mlp(BASE, **{name: OFF2}), INVALID, name)


def test_mlp_null_shape_and_no_tokens():
    refused(mlp(None), INVALID, "shape is NULL")
    none = dict.fromkeys(("x_q", "x_scales", "offsets", "w13_q", "w13_scales", "w2_q", "w2_scales", "y_perm"))
    assert mlp(BASE.replace(T=0), ws=None, ws_bytes=0, **none) == (moe.MOE_OK, "")


def test_mlp_workspace():
    for sh in (BASE, BASE.replace(T=8192, d=7168, F=2048), BASE.replace(expert_capacity=5)):
        n = moe.workspace_size(sh, moe.MOE_WS_MX_FFN)
        assert n % 256 == 0 and n >= sh.capacity * (sh.F + sh.F // 32)
    for sh in (BASE.replace(d=72), BASE.replace(F=40)):
        with pytest.raises(moe.MoEError, match="% 32"):
            moe.workspace_size(sh, moe.MOE_WS_MX_FFN)


# ---- few-token layer ----
DECODE = ("x", "w_router", "bias", "w13", "w13_scales", "w2", "w2_scales", "ws13", "ws13_scales", "ws2", "ws2_scales", "out")


def decode(sh, mx=False, ws=FAKE, ws_bytes=BIG, **ptr):
    ps = {n: FAKE for n in DECODE}
    ps["bias"] = None
    if not mx:
        ps.update(w13_scales=None, w2_scales=None, ws13_scales=None, ws2_scales=None)
    if sh is not None and not sh.F_shared:
        ps.update(ws13=None, ws13_scales=None, ws2=None, ws2_scales=None)
    ps.update(ptr)
    shape = None if sh is None else ctypes.byref(moe.shape_c(sh))
    return status(moe.lib().moe_layer_decode, shape, *(ps[n] for n in DECODE), ws, ws_bytes, None)


@pytest.mark.parametrize("change,kw,st,needle", [
    (dict(T=65), {}, UNSUPPORTED, "T (65) > 64"),
    (dict(T=-1), {}, INVALID, "T (-1) < 0"),
    (dict(d=60), {}, UNSUPPORTED, "d (60) % 8 != 0"),
    (dict(d=1 << 20), {}, UNSUPPORTED, ">= 2^20"),
    (dict(F=1 << 20), {}, UNSUPPORTED, ">= 2^20"),
    (dict(F_shared=1 << 20), {}, UNSUPPORTED, ">= 2^20"),
    (dict(d=72), dict(mx=True), UNSUPPORTED, "d (72) % 32 != 0"),
    (dict(F=40), dict(mx=True), UNSUPPORTED, "F (40) % 32 != 0"),
    (dict(F_shared=40), dict(mx=True), UNSUPPORTED, "F_shared (40) % 32 != 0"),
    (dict(d=16416), dict(mx=True), UNSUPPORTED, "d (16416) > 16384"),
    (dict(F=32800), dict(mx=True), UNSUPPORTED, "F (32800)"),
    (dict(F_shared=32800), dict(mx=True), UNSUPPORTED, "F_shared (32800)"),
    (dict(gate=wl.GATE_SIGMOID), dict(bias=FAKE), UNSUPPORTED, "bias"),
    ({}, dict(w13_scales=FAKE), INVALID, "scales are given for some"),
    ({}, dict(w2_scales=FAKE), INVALID, "scales are given for some"),
    (dict(F_shared=64), dict(mx=True, ws13_scales=None), INVALID, "scales are given for some"),
    (dict(F_shared=64), dict(ws2_scales=FAKE), INVALID, "scales are given for some"),
    (dict(F_shared=64), dict(ws13=None), INVALID, "ws13 is NULL"),
    (dict(F_shared=64), dict(ws2=OFF8), INVALID, "ws2"),
    ({}, dict(bias=OFF2), INVALID, "bias"),
    ({}, dict(ws=None), WORKSPACE, "workspace is NULL"),
    ({}, dict(ws_bytes=100), WORKSPACE, "required"),
])
def test_decode_refusals(change, kw, st, needle):
    refused(decode(BASE.replace(**change), **kw), st, needle)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("name", ["x", "w_router", "w13", "w2", "out"])
def test_decode_pointers(name, mx):
    refused(decode(BASE, mx, **{name: None}), INVALID, f"{name} is NULL")
    refused(decode(BASE, mx, **{name: OFF8}), INVALID, name)


def test_decode_misaligned_scales():
    for name in ("w13_scales", "w2_scales", "ws13_scales", "ws2_scales"):
        refused(decode(BASE.replace(F_shared=64), True, **{name: OFF8}), INVALID, name)


def test_decode_null_shape_and_no_tokens():
    refused(decode(None), INVALID, "shape is NULL")
    assert decode(BASE.replace(T=0), ws=None, ws_bytes=0, x=None, w_router=None, w13=None, w2=None,
                  out=None) == (moe.MOE_OK, "")


def test_decode_workspace():
    for sh in (BASE, BASE.replace(T=64, F_shared=2048), BASE.replace(T=1)):
        n = moe.workspace_size(sh, moe.MOE_WS_DECODE)
        slots = sh.T * sh.top_k
        assert n % 256 == 0 and n >= slots * (8 + 2 * sh.F + 4 * sh.d) + sh.T * (4 * sh.E + 2 * sh.F_shared)
    with pytest.raises(moe.MoEError, match="T \\(65\\)"):
        moe.workspace_size(BASE.replace(T=65), moe.MOE_WS_DECODE)
    # the chosen experts and gates lie where the layer's other workspaces have them
    assert moe.workspace_offset(BASE, moe.MOE_REGION_TOPK_IDX) == 0


# ---- wrappers: what the tensors are is checked before the library sees pointers ----
def test_wrappers_refuse_tensors_that_are_not_on_a_gpu():
    b, u = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4, 64), dtype=torch.uint8)
    for call in (lambda: moe.moe_mx_quantize(moe.MOE_MX_E4M3, b, u, u[:, :2]),
                 lambda: moe.moe_mx_dequantize(moe.MOE_MX_E4M3, u, u[:, :2], b),
                 lambda: moe.moe_add_rmsnorm(b, None, b[0], 1e-6, None, b),
                 lambda: moe.moe_add_rmsnorm_backward(b, None, b, b[0], b[:, 0].float(), b, b[0], u),
                 lambda: moe.moe_mx_grouped_ffn(BASE, moe.MOE_MX_E4M3, u, u, u, u, u, u, u, b, u),
                 lambda: moe.moe_layer_decode(BASE, b, b, None, b, b, None, None, b, u)):
        with pytest.raises(moe.MoEError, match="is on cpu, not on a GPU"):
            call()
    with pytest.raises(moe.MoEError, match="has 3 dimensions, expected 2"):
        moe.moe_mx_quantize(moe.MOE_MX_E4M3, b.view(2, 2, 64), u, u)


class _Pretend:
    """A host tensor that says that it is on a GPU: enough for the wrappers' checks, which look at nothing else."""

    def __init__(self, t, device="cuda:0"):
        self.t, self.is_cuda, self.device = t, True, torch.device(device)

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_wrappers_name_the_tensor_they_refuse():
    def p(shape, dtype=torch.bfloat16, device="cuda:0"):
        return _Pretend(torch.zeros(shape, dtype=dtype), device)
    u8 = torch.uint8
    x, q, s = p((4, 64)), p((4, 64), u8), p((4, 2), u8)
    bad = [p((4, 64), torch.float16), p((4, 32)), p((4, 64), device="cuda:1"), _Pretend(torch.zeros((64, 4)).bfloat16().t())]
    for b in bad:
        with pytest.raises(moe.MoEError, match="residual is .* expected contiguous torch.bfloat16"):
            moe.moe_add_rmsnorm(x, b, p(64), 1e-6, x, x)
    with pytest.raises(moe.MoEError, match="elements is"):
        moe.moe_mx_quantize(moe.MOE_MX_E2M1, x, q, s)
    with pytest.raises(moe.MoEError, match="scales is missing"):
        moe.moe_mx_quantize(moe.MOE_MX_E4M3, x, q, None)
    with pytest.raises(moe.MoEError, match="gamma is"):
        moe.moe_add_rmsnorm(x, None, p(32), 1e-6, None, x)
    with pytest.raises(moe.MoEError, match="rstd is"):
        moe.moe_add_rmsnorm_backward(x, None, x, p(64), p(4), x, p(64), q)
    sh = BASE.replace(T=4, top_k=2, d=64, F=32)
    cap = sh.capacity
    off = p(9, torch.int32)
    args = dict(x_q=p(cap * 64, u8), x_scales=p(cap * 2, u8), offsets=off, w13_q=p(8 * 32 * 64, u8), w13_scales=p(8 * 64 * 2, u8),
                w2_q=p(8 * 64 * 16, u8), w2_scales=p(8 * 64, u8), y_perm=p((cap, 64)), ws=p(1 << 20, u8))
    for name, wrong in (("x_q", p(cap * 64 - 1, u8)), ("x_scales", p(cap * 2 - 1, u8)), ("offsets", p(8, torch.int32)),
                        ("w13_q", p(8 * 32 * 64 - 1, u8)), ("w13_scales", p(8 * 64 * 2 - 1, u8)), ("w2_q", p(8 * 64 * 16 - 1, u8)),
                        ("w2_scales", p(8 * 64 - 1, u8)), ("y_perm", p((cap - 1, 64))), ("ws", p(64, torch.float32))):
        with pytest.raises(moe.MoEError, match=f"{name} is"):
            moe.moe_mx_grouped_ffn(sh, moe.MOE_MX_E4M3, **dict(args, **{name: wrong}))
    args = dict(x=p((4, 64)), w_router=p((8, 64)), bias=None, w13=p((8, 64, 64)), w2=p((8, 64, 32)), ws13=None, ws2=None,
                out=p((4, 64)), ws=p(1 << 20, u8))
    for name, wrong in (("x", p((3, 64))), ("w_router", p((7, 64))), ("bias", p(8)), ("w13", p((8, 32, 64))), ("w2", p((8, 32, 32))),
                        ("out", p((4, 64), torch.float32)), ("ws", p(64))):
        with pytest.raises(moe.MoEError, match=f"{name} is"):
            moe.moe_layer_decode(sh, **dict(args, **{name: wrong}))
    with pytest.raises(moe.MoEError, match="w13_scales is missing"):
        moe.moe_layer_decode(sh, **dict(args, w13=p(8 * 64 * 32, u8), w2=p(8 * 64 * 16, u8)), scales=(None,) * 4)


# ---- the host layer under the sanitizers ----
@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the ROCm headers")
def test_host_layer_under_asan_ubsan(tmp_path):
    """The entry points as plain host C++ with the launchers replaced, driven up to their launches."""
    exe = str(tmp_path / "abi_serving_sanitized")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
           os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_serving.cpp"), os.path.join(CSRC, "sizes.cpp"),
           os.path.join(HERE, "stubs.cpp"), os.path.join(HERE, "serving_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ALL OK"), r.stdout[-3000:] + r.stderr[-3000:]


def test_decode_on_4_bit_weights_that_were_not_made():
    layer = moe.DeviceLayer.__new__(moe.DeviceLayer)
    layer.shape, layer.w13, layer.w2, layer.ws13, layer.ws2, layer.ws_decode = BASE, None, None, None, None, object()
    with pytest.raises(moe.MoEError, match="quantize"):
        layer.decode(mx=True)
