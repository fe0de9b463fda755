"""Host side of the operators around the attention without a GPU: what the binding refuses (fake tensors, in a child process), the argument checks under
AddressSanitizer and UndefinedBehaviorSanitizer, and what the compiler gives the kernels."""
import glob
import os
import re
import shutil
import subprocess
import sys

import pytest

from paper_2512_07782_amd import build as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

REFUSALS = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2512_07782_amd as g

def refused(kind, text, f, *a, **kw):
    try:
        f(*a, **kw)
    except kind as e:
        assert text in str(e), (text, str(e))
        print("ok", flush=True)
    else:
        raise AssertionError(text)

with FakeTensorMode():
    new = lambda *s, dtype=torch.bfloat16, device="cuda:0": torch.empty(s, dtype=dtype, device=device)
    i32 = lambda *s, **kw: new(*s, dtype=torch.int32, **kw)
    f32 = lambda *s, **kw: new(*s, dtype=torch.float32, **kw)
    q, k = new(2, 9, 4, 64), new(2, 9, 2, 64)
    Q, K = new(2, 4, 9, 64), new(2, 2, 9, 64)
    rope = g.gfwa_qk_norm_rope
    refused(ValueError, "divide", rope, q, new(2, 9, 3, 64))
    refused(ValueError, "shape", rope, q, new(2, 8, 2, 64))
    refused(TypeError, "dtype", rope, q, f32(2, 9, 2, 64))
    refused(ValueError, "contiguous in its last", rope, new(2, 9, 64, 4).transpose(2, 3), k)
    refused(ValueError, "shape", rope, q, k, wq=f32(63))
    refused(TypeError, "dtype", rope, q, k, wq=new(64))
    refused(TypeError, "float64", rope, q, k, freq=f32(32))
    refused(ValueError, "rot / 2", rope, q, k, freq=new(2, 16, dtype=torch.float64))
    refused(ValueError, "norm=False", rope, q, k, wk=f32(64), norm=False)
    refused(ValueError, "shape", rope, q, k, pos=i32(9))
    refused(TypeError, "int32", rope, q, k, pos=new(2, 9, dtype=torch.int64))
    refused(ValueError, "is on cuda:1", rope, q, new(2, 9, 2, 64, device="cuda:1"))
    refused(ValueError, "is on cuda:1", rope, q, k, wq=f32(64, device="cuda:1"))
    refused(ValueError, "is on cuda:1", rope, q, k, Q=new(2, 4, 9, 64, device="cuda:1"))
    refused(ValueError, "GPU", rope, q, new(2, 9, 2, 64, device="cpu"))
    refused(TypeError, "unsupported dtype", rope, new(2, 9, 4, 64, dtype=torch.float16), k)
    back = g.gfwa_qk_norm_rope_backward
    refused(ValueError, "shape", back, q, k, Q, new(2, 4, 9, 64))
    refused(ValueError, "contiguous", back, q, k, new(2, 9, 4, 64).transpose(1, 2), K)
    refused(ValueError, "dv without dV", back, q, k, Q, K, dv=k)
    refused(ValueError, "norm=False", back, q, k, Q, K, norm=False, dwq=f32(64))
    refused(ValueError, "is on cuda:1", back, q, k, Q, new(2, 2, 9, 64, device="cuda:1"))
    refused(ValueError, "is on cuda:1", back, q, k, Q, K, wq=f32(64), workspace=new(9, dtype=torch.uint8, device="cuda:1"))
    Kp, cp, table = new(6, 2, 16, 64), f32(6, 4, 16), i32(3, 2)
    kr, qr, al, start, cached = new(7, 2, 64), new(7, 4, 64), f32(7, 4), i32(4), i32(3)
    app = g.gfwa_append_paged
    refused(ValueError, "shape", app, kr, new(7, 3, 64), Kp, Kp, start, cached, table)
    refused(ValueError, "shape", app, kr, kr, Kp, Kp, cached, cached, table)
    refused(ValueError, "shape", app, kr, kr, Kp, Kp, start, cached, i32(2, 2))
    refused(ValueError, "alpha without cp", app, kr, kr, Kp, Kp, start, cached, table, alpha=al)
    refused(ValueError, "divide", app, kr, kr, Kp, Kp, start, cached, table, q=new(7, 3, 64))
    refused(ValueError, "shape", app, kr, kr, Kp, Kp, start, cached, table, q=qr, alpha=f32(7, 2), cp=cp)
    refused(ValueError, "shape", app, kr, kr, Kp, Kp, start, cached, table, q=qr, alpha=al, cp=f32(6, 2, 16))
    refused(TypeError, "dtype", app, kr, kr, Kp, f32(6, 2, 16, 64), start, cached, table)
    refused(ValueError, "contiguous", app, kr, kr, new(6, 16, 2, 64).transpose(1, 2), Kp, start, cached, table)
    refused(ValueError, "is on cuda:1", app, kr, kr, Kp, Kp, start, i32(3, device="cuda:1"), table)
    dec = g.gfwa_decode_paged
    qd, pos = new(3, 4, 64), i32(3)
    refused(ValueError, "divide", dec, new(3, 3, 64), Kp, Kp, cp, table, pos, 4, 0.1)
    many = (1 << 32) + 3
    refused(ValueError, "too large", dec, new(many, 4, 64), Kp, Kp, cp, i32(many, 2), i32(many), 4, 0.1)
    refused(ValueError, "too large", app, kr, kr, Kp, Kp, i32(many + 1), i32(many), i32(many, 2))
    refused(ValueError, "too large", app, kr[:1].expand(many, 2, 64), kr[:1].expand(many, 2, 64), Kp, Kp, start, cached, table)
    refused(ValueError, "too large", rope, q[:1].expand(many, 9, 4, 64), k[:1].expand(many, 9, 2, 64))
    refused(TypeError, "cp", dec, qd, Kp, Kp, None, table, pos, 4, 0.1)
    refused(ValueError, "shape", dec, qd, Kp, Kp, cp, table, i32(4), 4, 0.1)
    refused(TypeError, "int32", dec, qd, Kp, Kp, cp, table, new(3, dtype=torch.int64), 4, 0.1)
    refused(ValueError, "contiguous", dec, new(4, 3, 64).transpose(0, 1), Kp, Kp, cp, table, pos, 4, 0.1)
    refused(ValueError, "is on cuda:1", dec, qd, Kp, Kp, cp, table, pos, 4, 0.1, o=new(3, 4, 64, device="cuda:1"))
print("all refused")
"""


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="for machines without a GPU")
def test_binding_refuses():
    r = subprocess.run([sys.executable, "-c", REFUSALS], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=ROOT,
                       env=dict(os.environ, PYTHONPATH=ROOT), timeout=300)
    assert r.returncode == 0 and "all refused" in r.stdout, r.stdout[-4000:]


def test_argument_checks_under_sanitizers(tmp_path):
    csrc, objdir = b.CSRC, os.path.join(b.HERE, "_build")
    others = [os.path.join(objdir, s.replace(".hip", ".o")) for s in b.SOURCES if s != "api.hip"]
    rt = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    if not os.path.exists(HIPCC) or not rt or not all(os.path.exists(o) for o in others):
        pytest.skip("no hipcc, no sanitizer runtime of its clang, or the library's objects are not built here")
    host = [x for kind in ("address", "undefined") for x in ("-Xarch_host", "-fsanitize=" + kind)] + ["-Xarch_host", "-fno-sanitize-recover=all"]
    obj, lib = str(tmp_path / "api.o"), str(tmp_path / "lib.so")
    subprocess.run([HIPCC] + b.FLAGS + ["-O1", "-g"] + host + ["-c", os.path.join(csrc, "api.hip"), "-o", obj], check=True, capture_output=True, timeout=600)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-shared-libsan", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-o", lib,
                    obj] + others, check=True, capture_output=True, timeout=600)
    env = dict(os.environ, LD_PRELOAD=rt[0], GFWA_LIB=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               PYTHONPATH=ROOT + os.pathsep + os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.join(ROOT, "tests", "test_layer_abi.py")], env=env, cwd=ROOT,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-4000:]


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc here")
@pytest.mark.parametrize("source", ["qk_norm_rope.hip", "append_paged.hip", "decode_paged.hip"])
def test_kernels_do_not_spill(source):
    cmd = [HIPCC] + b.FLAGS + b.EXTRA_FLAGS.get(source, []) + ["--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                                                               os.path.join(b.CSRC, source), "-o", os.devnull]
    said = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    scratch = dict(re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", said, re.S))
    assert scratch and not any(int(x) for x in scratch.values()), scratch


def test_bench_knows_the_paged_step():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--help"], stdout=subprocess.PIPE, text=True, check=True, timeout=120)
    assert "--paged PAGE" in r.stdout
