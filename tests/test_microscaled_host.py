"""Microscaled operands and the norm without a GPU: refusals of the C entry points and of the binding, and pins of the 64-bit
definitions that the GPU tests compare with."""
import ctypes
import inspect
import os
import re
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

from oracle import microscaled as mx
from paper_2502_05003_amd import binding as q
from paper_2502_05003_amd import build

from test_kernel_ordering import reads_outstanding_at_barriers

FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)   # never dereferenced: validation fails first, or nothing to do
OFF1, OFF2 = ctypes.c_void_p(0x10001), ctypes.c_void_p(0x10002)
OK, NULL, SHAPE, BLOCK, ALIGN, DTYPE, ARG = 0, 1, 2, 4, 5, 6, 8


@pytest.fixture(scope="module")
def lib():
    return q.load()


def test_quantizer_refuses(lib):
    def call(x=FAKE, dtype=1, rows=0, cols=512, ld=512, n=32, fmt=0, codes=FAKE, scales=FAKE, mask=FAKE):
        return lib.quest_hadamard_quantize_mx(x, dtype, rows, cols, ld, n, fmt, codes, scales, mask, None)
    assert call() == OK and call(mask=None) == OK and call(x=None, codes=None, scales=None) == OK and call(scales=OFF1) == OK
    for missing in ("x", "codes", "scales"):
        assert call(rows=4, **{missing: None}) == NULL
    assert call(dtype=2) == DTYPE and call(fmt=2) == DTYPE and call(fmt=-1) == DTYPE
    for cols in (0, 16, 31, 40, 16416, -32):
        assert call(cols=cols, ld=32768) == SHAPE
    assert call(rows=-1) == SHAPE and call(ld=480) == SHAPE and call(rows=1 << 24) == SHAPE
    assert call(rows=(1 << 24) - 1, cols=2048, ld=2048) == SHAPE          # more than 2^34 elements
    for n in (0, -1, 3, 48, 1024, 32768):
        assert call(n=n) == BLOCK
    assert call(cols=96, n=64) == BLOCK
    assert call(x=ODD) == ALIGN and call(codes=ODD) == ALIGN and call(mask=OFF1) == ALIGN and call(ld=516) == ALIGN
    assert call(ld=516, dtype=0) == OK and call(ld=518, dtype=0) == ALIGN


def test_reading_back_refuses(lib):
    def call(codes=FAKE, scales=FAKE, fmt=1, rows=0, cols=512, out=FAKE, dtype=1, ld=512):
        return lib.quest_dequantize_mx(codes, scales, fmt, rows, cols, out, dtype, ld, None)
    assert call() == OK and call(codes=None) == OK
    assert call(rows=1, codes=None) == NULL and call(rows=1, scales=None) == NULL and call(rows=1, out=None) == NULL
    assert call(fmt=3) == DTYPE and call(dtype=5) == DTYPE
    assert call(cols=48) == SHAPE and call(ld=511) == SHAPE and call(rows=-3) == SHAPE
    assert call(codes=ODD) == ALIGN and call(out=OFF2) == ALIGN and call(ld=516) == ALIGN


def test_product_refuses(lib):
    def call(a=FAKE, sa=FAKE, fmt=1, M=0, b=FAKE, sb=FAKE, N=8, K=512, y=FAKE, ld=8, acc=None):
        return lib.quest_lowbit_gemm_mx(a, sa, fmt, M, b, sb, N, K, y, ld, acc, None)
    assert call() == OK and call(M=8, N=0, ld=0) == OK and call(y=None) == OK and call(a=None) == OK
    for missing in ("a", "sa", "b", "sb", "y"):
        assert call(M=4, **{missing: None}) == NULL
    assert call(fmt=2) == DTYPE
    for K in (0, 64, 192, 65536 + 128, -128):
        assert call(K=K) == SHAPE
    assert call(M=-1) == SHAPE and call(N=-1) == SHAPE and call(M=(1 << 22) + 1) == SHAPE and call(N=(1 << 22) + 1) == SHAPE
    assert call(ld=7) == SHAPE and call(ld=7, y=None, acc=FAKE) == OK
    assert call(a=ODD) == ALIGN and call(b=ODD) == ALIGN and call(sa=OFF2) == ALIGN and call(sb=OFF1) == ALIGN
    assert call(y=OFF1) == ALIGN and call(acc=OFF2) == ALIGN and call(y=OFF2) == OK


def test_gradient_products_refuse(lib):
    def call(which=0, dy=FAKE, c=FAKE, s=FAKE, fmt=0, M=512, N=256, K=512, out=FAKE, ws=FAKE, wsb=1 << 30):
        return lib.quest_grad_gemm_mx(which, dy, c, s, fmt, M, N, K, out, ws, wsb, None)
    for missing in ("dy", "c", "s", "out"):
        assert call(**{missing: None}) == NULL
    assert call(which=2) == ARG and call(which=-1) == ARG and call(fmt=2) == DTYPE
    assert call(M=520) == SHAPE and call(N=32) == SHAPE and call(K=96) == SHAPE and call(M=1 << 23) == SHAPE and call(M=-64) == SHAPE
    need = q.quest_grad_gemm_mx_workspace_bytes(0, 512, 256, 512)
    assert need == 256 * 512 * 2 and q.quest_grad_gemm_mx_workspace_bytes(0, 64, 256, 512) == 0
    assert q.quest_grad_gemm_mx_workspace_bytes(0, 96, 256, 512) == -1
    assert call(M=0) == OK and call(which=1, N=0, ws=None, wsb=0) == OK
    assert call(M=0, dy=None, out=None) == OK and call(which=1, N=0, dy=None, out=None, ws=None, wsb=0) == OK
    assert call(N=0, out=None) == NULL and call(which=1, M=0, out=None) == NULL      # a sum over nothing is written, too
    assert q.quest_grad_gemm_mx_workspace_bytes(2, 512, 256, 512) == -1
    assert call(ws=None, wsb=0) == ARG and call(wsb=need - 1) == ARG and call(wsb=-1) == ARG
    assert call(dy=ODD) == ALIGN and call(c=ODD) == ALIGN and call(out=ODD) == ALIGN and call(ws=ODD) == ALIGN


@pytest.mark.parametrize("source", ["mx_tiles_e2m1.hip", "mx_tiles_e4m3.hip"])
def test_tiles_have_their_reads_back_at_barriers(source, tmp_path):
    """The transfers behind a barrier refill the stage that was read ahead of it, so no wave may arrive with LDS reads on their way."""
    out = tmp_path / "kernels.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.HIPCC_FLAGS, *build.EXTRA_FLAGS.get(source, []),
                    "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    found = {k: v for k, v in reads_outstanding_at_barriers(out.read_text()).items() if "mx_tile_kernel" in k}
    assert len(found) >= 4 and all(len(v) >= 3 for v in found.values())
    assert {k: v for k, v in found.items() if any(v)} == {}
    counted = 0
    for kernel, waits in waits_at_barriers(out.read_text()).items():
        if "mx_tile_kernel" in kernel:
            assert all(allowed is not None and allowed <= stores for allowed, stores in waits), kernel
            counted += sum(allowed > 0 for allowed, _ in waits)
    assert counted >= 3      # tiles of 256: where one begins and where one ends; of 128: where one begins


def waits_at_barriers(assembly):
    """{kernel: [(memory operations that the last wait ahead of a barrier leaves on their way, stores between it and the last
    transfer into LDS ahead of it)]}: with as many stores behind the transfers as are left, the transfers have landed."""
    found, kernel, stores, last = {}, None, 0, None
    for line in assembly.splitlines():
        line = line.split(";")[0].strip()
        label = re.match(r"(_Z\w+):", line)
        if label:
            kernel, stores, last = label.group(1), 0, None
            found[kernel] = []
        elif line.startswith("buffer_load") and line.endswith("lds"):
            stores, last = 0, None
        elif line.startswith("buffer_store"):
            stores += 1
        elif line.startswith("s_waitcnt"):
            wait = re.search(r"vmcnt\((\d+)\)", line)
            if wait and (last is None or int(wait.group(1)) <= last[0]):
                last = (int(wait.group(1)), stores)
        elif line.startswith("s_barrier"):
            found[kernel].append(last or (None, stores))
            last = None
    return found


def test_the_waits_on_a_sample():
    sample = """
_Zk:
	buffer_load_dwordx4 v1, s[0:3], 0 offen lds
	buffer_store_dwordx4 v[2:5], v6, s[4:7], 0 offen
	s_waitcnt vmcnt(1)
	s_barrier
	buffer_load_dwordx4 v1, s[0:3], 0 offen offset:1024 lds
	s_waitcnt lgkmcnt(0)
	s_barrier
"""
    assert waits_at_barriers(sample) == {"_Zk": [(1, 1), (None, 0)]}


def test_norm_refuses(lib):
    def call(x=FAKE, ldx=512, r=FAKE, ldr=512, dtype=1, w=FAKE, wd=0, rows=0, cols=512, eps=1e-5, h=FAKE, y=FAKE, n=32, fmt=1,
             codes=FAKE, scales=FAKE, mask=FAKE, rstd=FAKE):
        return lib.quest_rms_norm_mx(x, ldx, r, ldr, dtype, w, wd, rows, cols, eps, h, y, n, fmt, codes, scales, mask, rstd, None)
    assert call() == OK and call(r=None, h=None, ldr=0) == OK and call(y=None, mask=None, rstd=None) == OK
    none = dict(codes=None, scales=None, mask=None)
    assert call(n=0, fmt=9, **none) == OK                       # not looked at without codes
    assert call(rows=1, y=None, **none) == NULL and call(rows=1, x=None) == NULL and call(w=None) == NULL
    assert call(dtype=2) == DTYPE and call(wd=2) == DTYPE and call(fmt=2) == DTYPE
    assert call(cols=48) == SHAPE and call(ldx=511) == SHAPE and call(ldr=480) == SHAPE and call(rows=-1) == SHAPE
    assert call(rows=1 << 24) == SHAPE
    assert call(n=24) == BLOCK and call(cols=2048, ldx=2048, ldr=2048, n=1024) == BLOCK and call(cols=96, n=64) == BLOCK
    for eps in (-1e-5, float("nan"), float("inf")):
        assert call(eps=eps) == ARG
    assert call(h=None) == ARG and call(r=None) == ARG          # the residual and what comes of it: both or neither
    assert call(scales=None) == ARG and call(codes=None) == ARG and call(codes=None, scales=None) == ARG
    for at in ("x", "r", "w", "h", "y", "codes", "mask"):
        assert call(**{at: ODD}) == ALIGN
    assert call(rstd=OFF2) == ALIGN and call(ldx=516) == ALIGN and call(ldr=516) == ALIGN and call(scales=OFF1) == OK


def test_norm_backward_refuses(lib):
    def call(dy=FAKE, h=FAKE, dtype=1, w=FAKE, wd=0, rstd=FAKE, dh=FAKE, rows=8, cols=512, dx=FAKE, dw=FAKE, ws=FAKE, wsb=1 << 30):
        return lib.quest_rms_norm_backward(dy, h, dtype, w, wd, rstd, dh, rows, cols, dx, dw, ws, wsb, None)
    for missing in ("dy", "h", "w", "rstd", "dx"):
        assert call(**{missing: None}) == NULL
    assert call(rows=0, dy=None, h=None, rstd=None, dx=None, dw=None) == OK
    assert call(dtype=3) == DTYPE and call(wd=-1) == DTYPE
    assert call(cols=40) == SHAPE and call(rows=-1) == SHAPE
    need = q.quest_rms_norm_backward_workspace_bytes(8, 512)
    assert need > 0 and q.quest_rms_norm_backward_workspace_bytes(8, 40) == -1 and q.quest_rms_norm_backward_workspace_bytes(-1, 64) == -1
    assert call(ws=None, wsb=0) == ARG and call(wsb=need - 1) == ARG and call(wsb=-1) == ARG
    for at in ("dy", "h", "w", "dh", "dx", "dw", "ws"):
        assert call(**{at: ODD}) == ALIGN
    assert call(rstd=OFF2) == ALIGN


# ---- the binding's own checks (tensors on the CPU: everything else is refused before the place is looked at)

def u8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def test_binding_refuses_other_shapes_types_and_places():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    good = dict(codes=u8(4, 32), scales=u8(4, 2), mask=u8(4, 8))
    for changed in (dict(codes=u8(4, 64)), dict(codes=u8(4, 64)[:, ::2]), dict(scales=u8(4, 1)), dict(scales=torch.zeros(4, 2)),
                    dict(mask=u8(4, 4)), dict(codes=u8(128))):
        with pytest.raises(ValueError):
            q.quest_hadamard_quantize_mx(x, 32, q.QUEST_MX_E2M1, **(good | changed))
    with pytest.raises(ValueError, match="format"):
        q.quest_hadamard_quantize_mx(x, 32, 7, **good)
    with pytest.raises(ValueError, match="not contiguous"):
        q.quest_hadamard_quantize_mx(torch.zeros(64, 4, dtype=torch.bfloat16).t(), 32, q.QUEST_MX_E2M1, **good)
    with pytest.raises(ValueError):
        q.quest_hadamard_quantize_mx(x[0], 32, q.QUEST_MX_E2M1, **good)
    with pytest.raises(ValueError):
        q.quest_dequantize_mx(u8(4, 32), u8(4, 2), q.QUEST_MX_E2M1, out=torch.zeros(4, 128))
    a, s, b, t = u8(4, 128), u8(4, 4), u8(6, 64), u8(6, 4)
    y = torch.zeros(4, 6, dtype=torch.bfloat16)
    for args in ((a[:, :64], s, 1, b, t, 128), (a, s[:, :3], 1, b, t, 128), (a, s, 0, b, t, 128), (a, s, 1, u8(6, 128), t, 128)):
        with pytest.raises(ValueError):
            q.quest_lowbit_gemm_mx(*args, y=y)
    with pytest.raises(ValueError):
        q.quest_lowbit_gemm_mx(a, s, 1, b, t, 128, y=torch.zeros(6, 4, dtype=torch.bfloat16).t())
    with pytest.raises(TypeError):
        q.quest_lowbit_gemm_mx(a, s, 1, b, t, 128, y=torch.zeros(4, 6))
    with pytest.raises(ValueError):
        q.quest_lowbit_gemm_mx(a, s, 1, b, t, 128, y=None, acc_out=torch.zeros(4, 7))
    dy = torch.zeros(128, 192, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        q.quest_grad_gemm_mx(0, dy, u8(192, 64), u8(192, 4), 0, 128, 192, 128, out=torch.zeros(192, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        q.quest_grad_gemm_mx(1, dy, u8(192, 64), u8(192, 4), 0, 128, 192, 128, out=torch.zeros(192, 128, dtype=torch.bfloat16))
    w, rstd = torch.zeros(64), torch.zeros(4)
    with pytest.raises(TypeError):
        q.quest_rms_norm_mx(x, w, 1e-5, residual=x.float(), h_out=x.clone(), y_out=x.clone())
    for changed in (dict(y_out=x.float()), dict(residual=x[:2], h_out=x), dict(rstd=rstd[:3], y_out=x), dict(y_out=x[:, :32])):
        with pytest.raises(ValueError):
            q.quest_rms_norm_mx(x, w, 1e-5, **changed)
    with pytest.raises(ValueError):
        q.quest_rms_norm_mx(x, w[:32], 1e-5, y_out=x.clone())
    for changed in (dict(dx=x.float()), dict(dweight=w.double()), dict(dh=x[:, ::2]), dict(dh=x[:3])):
        with pytest.raises(ValueError):
            q.quest_rms_norm_backward(x, x, w, rstd, **(dict(dx=x.clone(), dweight=w.clone()) | changed))


def test_binding_refuses_tensors_elsewhere(monkeypatch):
    """Host memory must not reach a kernel."""
    monkeypatch.setattr(q, "_current_device", lambda: 0)
    x, w, rstd = torch.zeros(128, 128, dtype=torch.bfloat16), torch.zeros(128), torch.zeros(128)
    codes, scales = u8(128, 64), u8(128, 4)
    for call in (lambda: q.quest_hadamard_quantize_mx(x, 32, 0, codes=codes, scales=scales),
                 lambda: q.quest_dequantize_mx(codes, scales, 0, out=x),
                 lambda: q.quest_lowbit_gemm_mx(codes, scales, 0, codes, scales, 128, y=x),
                 lambda: q.quest_grad_gemm_mx(0, x, codes, scales, 0, 128, 128, 128, out=x),
                 lambda: q.quest_rms_norm_mx(x, w, 1e-5, 32, 0, codes=codes, scales=scales),
                 lambda: q.quest_rms_norm_backward(x, x, w, rstd, dx=x, dweight=None)):
        with pytest.raises(ValueError, match="is on cpu"):
            call()


# ---- the two ways to an entry point, native code and ctypes (stand-ins record what they are given)

def mx_calls(dtype):
    """name, positional, keyword arguments: forms and options of every call; tensors in host memory"""
    x, wide, w = torch.zeros(4, 64, dtype=dtype), torch.zeros(4, 96, dtype=dtype), torch.zeros(64)
    quantized = dict(codes=u8(4, 32), scales=u8(4, 2))
    yield "quest_hadamard_quantize_mx", (x, 32, 0), quantized
    yield "quest_hadamard_quantize_mx", (wide[:, :64], 1, 1), dict(codes=u8(4, 64), scales=u8(4, 2), mask=u8(4, 8))
    yield "quest_hadamard_quantize_mx", (wide[1:2, :64], 1, 0), dict(codes=u8(1, 32), scales=u8(1, 2))
    yield "quest_hadamard_quantize_mx", (x[:0], 1, 0), dict(codes=u8(0, 32), scales=u8(0, 2))
    yield "quest_dequantize_mx", (u8(4, 32), u8(4, 2), 0), dict(out=wide[:, :64])
    a, s, b, t, y = u8(4, 128), u8(4, 4), u8(6, 64), u8(6, 4), torch.zeros(4, 9, dtype=torch.bfloat16)
    yield "quest_lowbit_gemm_mx", (a, s, 1, b, t, 128), dict(y=y[:, :6])
    yield "quest_lowbit_gemm_mx", (a[:, :64].contiguous(), s, 0, b, t, 128), dict(y=None, acc_out=torch.zeros(4, 6))
    dy, scratch = torch.zeros(128, 192, dtype=torch.bfloat16), torch.zeros(33, dtype=torch.int16)
    yield "quest_grad_gemm_mx", (0, dy, u8(192, 64), u8(192, 4), 0, 128, 192, 128), dict(out=torch.zeros(128, 128, dtype=torch.bfloat16))
    yield ("quest_grad_gemm_mx", (1, dy, u8(128, 128), u8(128, 4), 1, 128, 192, 128),
           dict(out=torch.zeros(192, 128, dtype=torch.bfloat16), workspace=scratch))
    yield "quest_rms_norm_mx", (x, w, 1e-5, 32, 0), quantized
    yield ("quest_rms_norm_mx", (wide[:, :64], w.bfloat16(), 1e-6, 1, 1),
           dict(codes=u8(4, 64), scales=u8(4, 2), mask=u8(4, 8), residual=wide[:, 32:], h_out=x, y_out=x.clone(), rstd=torch.zeros(4)))
    yield "quest_rms_norm_mx", (x, w, 1e-5), dict(y_out=x.clone())
    yield "quest_rms_norm_backward", (x, x, w, torch.zeros(4)), dict(dx=x.clone(), dweight=None)
    yield ("quest_rms_norm_backward", (x, x, w.bfloat16(), torch.zeros(4)),
           dict(dx=x.clone(), dweight=w.clone(), dh=x.clone(), workspace=scratch))


@pytest.fixture
def record(monkeypatch):
    seen, keep = [], {}
    real = q.load()

    def entry(name):
        def called(*args):
            seen.append((name, args))
            return 0
        return ctypes.CFUNCTYPE(ctypes.c_int, *getattr(real, name).argtypes)(called)
    keep.update({name: entry(name) for name in q._MX_NATIVE})
    from paper_2502_05003_amd import quest_python
    native = quest_python.MxCalls(*(ctypes.cast(f, ctypes.c_void_p).value for f in keep.values()))
    refuses = types.SimpleNamespace(**{name: lambda *args: None for name in dir(native) if not name.startswith("_")})
    library = types.SimpleNamespace(mx_calls=native, quest_status_string=real.quest_status_string, **keep)
    monkeypatch.setattr(q, "_lib", library)
    monkeypatch.setattr(q, "_stream", lambda: 0x7fff_1234_5678)
    monkeypatch.setattr(q, "_current_device", lambda: -1)          # what tensors in host memory say
    return types.SimpleNamespace(seen=seen, native=native, refuses=refuses, library=library, keep=keep)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_ways_pass_the_same_arguments(record, dtype):
    named = set()
    for name, args, kwargs in mx_calls(dtype):
        record.library.mx_calls = record.native
        assert getattr(q, name)(*args, **kwargs) is None
        record.library.mx_calls = record.refuses
        getattr(q, name)(*args, **kwargs)
        native, general = record.seen[-2:]
        assert native[0] == general[0] == name and native[1] == general[1], name
        named.add(name)
    assert named == set(q._MX_NATIVE) and len(record.seen) % 2 == 0


def test_a_workspace_is_as_large_as_it_says(record, monkeypatch):
    """One whose elements share or skip memory has fewer bytes, or others' among them."""
    x, w, rstd = torch.zeros(128, 128, dtype=torch.bfloat16), torch.zeros(128), torch.zeros(128)
    for workspace in (u8(1).expand(1 << 20), u8(1 << 12)[::2], torch.zeros(64, 32).t()):
        for calls in (record.native, record.refuses):
            record.library.mx_calls = calls
            with pytest.raises(ValueError, match="workspace"):
                q.quest_grad_gemm_mx(0, x, u8(128, 64), u8(128, 4), 0, 128, 128, 128, out=x.clone(), workspace=workspace)
            with pytest.raises(ValueError, match="workspace"):
                q.quest_rms_norm_backward(x, x, w, rstd, dx=x.clone(), dweight=w.clone(), workspace=workspace)
    assert not record.seen


@pytest.mark.parametrize("fmt,block", [(9, 32), (-1, 0), (1, 7)])
def test_norm_without_codes_looks_at_no_format_and_block(record, fmt, block):
    """The library does not look at them then; both ways pass them on."""
    x, w, rstd = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64), torch.zeros(4)
    for calls in (record.native, record.refuses):
        record.library.mx_calls = calls
        q.quest_rms_norm_mx(x, w, 1e-5, block, fmt, y_out=x.clone(), rstd=rstd)
    (_, native), (_, general) = record.seen
    at = record.keep["quest_rms_norm_mx"].argtypes.index(ctypes.c_float)
    for args in (native, general):
        assert args[at + 3:at + 8] == (block, fmt, None, None, None)
    record.library.quest_rms_norm_mx = None                        # native alone
    record.library.mx_calls = record.native
    q.quest_rms_norm_mx(x, w, 1e-5, block, fmt, y_out=x.clone())
    assert len(record.seen) == 3
    for outputs in (dict(codes=u8(4, 64), scales=u8(4, 2)), dict(codes=u8(4, 32), scales=u8(4, 2))):
        if fmt not in (0, 1):
            with pytest.raises(ValueError, match="format"):
                q.quest_rms_norm_mx(x, w, 1e-5, block, fmt, **outputs)


def test_plain_calls_are_native_ones(record):
    for name in q._MX_NATIVE:
        setattr(record.library, name, None)
    for name, args, kwargs in mx_calls(torch.bfloat16):
        getattr(q, name)(*args, **kwargs)
    assert len(record.seen) == len(list(mx_calls(torch.bfloat16)))


def test_what_is_refused_reaches_no_entry_point(record, monkeypatch):
    """The native way gives the calls of the tests above to the general one, which raises."""
    test_binding_refuses_other_shapes_types_and_places()
    monkeypatch.setattr(q, "_current_device", lambda: 0)
    for name, args, kwargs in mx_calls(torch.bfloat16):
        with pytest.raises(ValueError, match="is on cpu"):
            getattr(q, name)(*args, **kwargs)

    def fails():
        raise RuntimeError("no device")
    monkeypatch.setattr(q, "_current_device", fails)
    for name, args, kwargs in mx_calls(torch.bfloat16):
        with pytest.raises(RuntimeError, match="no device"):
            getattr(q, name)(*args, **kwargs)
    assert not record.seen


def fewer_addresses(*addresses):
    raise TypeError("one address for each entry point")


@pytest.mark.parametrize("kinds", [dict(), dict(MxCalls=fewer_addresses)])
def test_with_a_native_module_of_other_entry_points_calls_take_the_general_way(kinds, record, monkeypatch):
    """One built for this torch, but from other sources: without these calls, or with another number of them."""
    import paper_2502_05003_amd as package
    from paper_2502_05003_amd import quest_python
    module = types.SimpleNamespace(TORCH_BUILD=q.torch_build(), Calls=quest_python.Calls, **kinds)
    monkeypatch.setattr(package, "quest_python", module)
    monkeypatch.setitem(sys.modules, package.__name__ + ".quest_python", module)
    monkeypatch.setattr(q, "_lib", None)
    with pytest.warns(RuntimeWarning, match="g.build()"):
        assert q.quest_container_bits(4) == 4
    record.library.mx_calls = q.load().mx_calls
    monkeypatch.setattr(q, "_lib", record.library)
    for name, args, kwargs in mx_calls(torch.bfloat16):
        getattr(q, name)(*args, **kwargs)
        assert record.seen[-1][0] == name


SIGNATURES = {
    "quest_hadamard_quantize_mx": ("x had_block fmt", "codes scales mask=None"),
    "quest_dequantize_mx": ("codes scales fmt", "out"),
    "quest_lowbit_gemm_mx": ("a_codes a_scales a_format b_codes b_scales K", "y acc_out=None"),
    "quest_grad_gemm_mx": ("which dy q_codes q_scales q_format M N K", "out workspace=None"),
    "quest_rms_norm_mx": ("x weight eps had_block=1 fmt=1",
                          "codes=None scales=None mask=None residual=None h_out=None y_out=None rstd=None"),
    "quest_rms_norm_backward": ("dy h weight rstd", "dx dweight dh=None workspace=None"),
}


def test_signatures():
    assert set(q._MX_NATIVE) == set(SIGNATURES)
    for name, expected in SIGNATURES.items():
        kinds = {inspect.Parameter.POSITIONAL_OR_KEYWORD: [], inspect.Parameter.KEYWORD_ONLY: []}
        for p in inspect.signature(getattr(q, name)).parameters.values():
            kinds[p.kind].append(p.name if p.default is p.empty else f"{p.name}={p.default}")
        assert tuple(" ".join(names) for names in kinds.values()) == expected, name


# ---- the definitions

def test_element_grids():
    assert mx.MAGNITUDES[0].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx.MAGNITUDES[1], e4m3) and mx.TRUSTED == (7.0, 464.0)


def test_hand_checked_group():
    g = np.zeros((1, 32))
    g[0, :12] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -5, -6, 0.3]
    code, scales, trust = mx.quantize(g, 0)
    assert scales[0, 0] == 127 and trust.all()
    assert code[0, :13].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 8, 14, 15, 1, 0]
    code, scales, trust = mx.quantize(g * 1.25, 0)                 # 7.5: clipped, beyond the trust border; 6.25 is within it
    assert scales[0, 0] == 127 and code[0, :2].tolist() == [7, 7] and trust[0, :3].tolist() == [False, True, True]
    code, scales, _ = mx.quantize(g * 4 / 3, 0)                    # 8: the next binade
    assert scales[0, 0] == 128 and code[0, 0] == 6
    zero = mx.quantize(np.zeros((1, 32)), 1)
    assert zero[1][0, 0] == 0 and not zero[0].any() and zero[2].all()
    g[0, 3] = np.nan
    code, scales, trust = mx.quantize(np.concatenate([g, g * 0 + 1], axis=1), 1)
    assert scales[0].tolist() == [255, 255] and not trust.any()


@pytest.mark.parametrize("fmt", [0, 1])
def test_quantized_values_are_the_nearest(fmt):
    x = np.random.default_rng(fmt).standard_normal((64, 96))
    code, scales, trust = mx.quantize(x, fmt)
    v = mx.values(mx.pack(code, fmt), scales, fmt)
    scale = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=1)
    grid = np.concatenate([mx.MAGNITUDES[fmt], -mx.MAGNITUDES[fmt]])
    for r in range(8):
        assert np.allclose(np.abs(v[r] - x[r]), np.abs(grid[:, None] * scale[r] - x[r]).min(0), rtol=1e-12, atol=1e-300)
    largest = np.abs(x).reshape(64, 3, 32).max(-1)
    top = mx.MAGNITUDES[fmt][-1]
    assert np.all(largest / np.ldexp(1.0, scales.astype(int) - 127) < 2.0 ** (mx.LARGEST_EXPONENT[fmt] + 1))
    assert np.all(np.abs(v)[~trust] == (top * scale)[~trust])


def test_transform_in_fp32_is_the_transform():
    from oracle import quest_oracle as qo
    x = np.random.default_rng(0).standard_normal((3, 512)).astype(np.float32)
    for n in (1, 2, 32, 512):
        assert np.allclose(mx.hadamard_f32(x, n), qo.hadamard(x.astype(np.float64), n), rtol=0, atol=2e-6)


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(3)
    h, w, dy = rng.standard_normal((2, 32)), rng.standard_normal(32), rng.standard_normal((2, 32))
    dx, dw = mx.rms_norm_backward(dy, h, w, mx.rms_norm(h, w, 1e-3)[1])
    loss = lambda a, b: (dy * mx.rms_norm(a, b, 1e-3)[0]).sum()  # noqa: E731
    for j in range(0, 32, 5):
        step = np.zeros((2, 32))
        step[1, j] = 1e-6
        assert dx[1, j] == pytest.approx((loss(h + step, w) - loss(h - step, w)) / 2e-6, rel=1e-6, abs=1e-8)
        assert dw[j] == pytest.approx((loss(h, w + step[1]) - loss(h, w - step[1])) / 2e-6, rel=1e-6, abs=1e-8)


def test_workgroup_memory_read_in_16_bytes_is_aligned_to_them():
    """A dynamic array begins behind the kernel's static ones, at a multiple of its own alignment and no more."""
    seen = 0
    for name in sorted(os.listdir(build.CSRC)):
        text = open(os.path.join(build.CSRC, name)).read()
        for declared, array in re.findall(r"extern __shared__ (.*?)(\w+)\[\];", text):
            wide = re.search(r"reinterpret_cast<[^<>]*(?:4|v4f|v4u)\s*\*>\([^;]*\b%s\b" % array, text)
            wide = wide or re.search(r"(?:load8|store8)\([^;]*\b%s\b" % array, text)
            if wide:
                seen += 1
                assert "aligned(16)" in declared, (name, array)
    assert seen >= 3


def test_quest_init_prepares_files_whose_launches_stand_in_headers():
    """A source file with kernels of its own has one set-up function, which quest_init calls, wherever the launches are written."""
    def with_headers(name, seen):
        if name in seen or not os.path.exists(os.path.join(build.CSRC, name)):
            return ""
        seen.add(name)
        text = re.sub(r"//.*", "", open(os.path.join(build.CSRC, name)).read())
        return text + "".join(with_headers(h, seen) for h in re.findall(r'#include "(\w+\.h)"', text))

    init = open(os.path.join(build.CSRC, "quest_api.hip")).read().split("quest_status quest_init(void)")[1]
    called = set(re.findall(r"quest::(prepare_\w+)\(\)", init))
    defined, in_headers = set(), 0
    for name in build.SOURCES:
        own = open(os.path.join(build.CSRC, name)).read()
        if "hipLaunchKernelGGL(" in with_headers(name, set()):
            setup = re.findall(r"^hipError_t (prepare_\w+_kernels)\(\)", own, flags=re.M)
            assert len(setup) == 1, f"{name}: set-up functions {setup}"
            defined.update(setup)
            in_headers += "hipLaunchKernelGGL(" not in own
    assert called == defined and in_headers >= 4


# ---- which kernel a product gets

def mx_plan(M, N, K):
    import plan
    ask = q.load().quest_plan_mx_gemm
    ask.argtypes, ask.restype = [ctypes.c_int64] * 3, plan._Plan
    p = ask(M, N, K)
    return {plan.FEW: "few", plan.TILES: "tiles"}[p.kernel], p.block_rows, p.block_cols


def test_products_reach_every_kernel():
    """The shapes of the GPU tests cover all blocks; short contractions and few rows keep off the tiles."""
    import test_gpu_microscaled as gpu
    reached = {mx_plan(*shape) for shape in gpu.PRODUCTS + gpu.LARGE_PRODUCTS}
    assert reached == {("few", 16, 16), ("few", 16, 32), ("few", 32, 32), ("few", 64, 32), ("few", 64, 64), ("tiles", 128, 128),
                       ("tiles", 256, 256)}
    for block in (128, 256):        # with workgroups that go on to another tile, and contractions of two stages, of whole ones and a half
        of = [s for s in gpu.LARGE_PRODUCTS if mx_plan(*s)[1] == block]
        assert any(-(-M // block) * -(-N // block) > 256 for M, N, K in of)
        assert {K % 256 for M, N, K in of} == {0, 128} and {384, 512} <= {K for M, N, K in of}
    assert mx_plan(1, 1 << 22, 65536)[0] == "few" and mx_plan(1 << 22, 1 << 22, 256) == ("few", 64, 64)
    assert mx_plan(1 << 22, 1 << 22, 384) == ("tiles", 256, 256)


def test_products_of_several_chunks_of_scales_reach_both_tiles():
    """Scales are staged 512 elements at a time: each remainder by that, with more than one chunk, with both blocks, in the
    workgroups' first tiles and in further ones."""
    import test_gpu_microscaled as gpu
    for block in (128, 256):
        of = [s for s in gpu.LARGE_PRODUCTS + gpu.CHUNKED_PRODUCTS if mx_plan(*s) == ("tiles", block, block) and s[2] > 512]
        assert {K % 512 for _, _, K in of} == {0, 128, 256, 384}
        for tiles_of_a_workgroup in (False, True):
            assert any(K % 512 == 384 and (-(-M // block) * -(-N // block) > 256) == tiles_of_a_workgroup for M, N, K in of), block


# what the kernel does with the header: transfers into two buffers of a chunk in turn, reads of a dword or of an aligned pair
STAGES = r"""
#include <stdio.h>
#include "mx_stages.h"

template <int STEPS>
int check()
{
    typedef quest::MxStages<STEPS> S;
    int bad = 0;
    for (int K = 384; K <= 65536; K += 128) {
        const int units = K / 128, stages = S::count(K);
        bad += stages < 2 || (stages - 1) * S::kStageK >= K || stages * S::kStageK < K || S::ends_in_half(K) != (units % STEPS != 0);
        int held = -1;
        for (int at = 0; at < stages; ++at) {
            if (S::opens_chunk(at))
                held = S::chunk(at);
            bad += held != S::chunk(at) || S::chunk(at) >= units;          // (its first dword is one of the row's)
            bad += S::word(at) % STEPS != 0 || S::word(at) + STEPS > S::kChunk;
            const int real = at == stages - 1 && S::ends_in_half(K) ? 1 : STEPS;
            for (int t = 0; t < real; ++t)
                bad += held + S::word(at) + t != at * STEPS + t || at * STEPS + t >= units;
            if (at == stages - 1)
                bad += at * STEPS + real != units;
        }
        bad += S::chunk(0) != 0 || !S::opens_chunk(0);                     // a tile's first stage
    }
    return bad;
}

int main()
{
    printf("%d %d\n", check<1>(), check<2>());
    return 0;
}
"""


def test_stages_find_their_scales(tmp_path):
    """All contractions that tiles take: each stage reads its own scale dwords, out of the chunk that the transfers left last."""
    source, program = tmp_path / "check.hip", str(tmp_path / "check")
    source.write_text(STAGES)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", build.CSRC,
                    str(source), "-o", program], check=True, capture_output=True)
    assert subprocess.run([program], check=True, capture_output=True, text=True).stdout.split() == ["0", "0"]
