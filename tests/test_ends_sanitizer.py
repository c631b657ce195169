"""The host side of the calls at the ends of a step (argument checks, plans of tensor lists and workspace sizes up to the first HIP call) rebuilt with the
undefined-behaviour sanitizer and swept through the C ABI without a GPU, every answer compared with the regular library's."""
import glob
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2410_08661_amd import build as qbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ["ends_api", "logprob", "heads", "adamw"]

CHILD = textwrap.dedent('''
    import ctypes as C, itertools, sys
    from paper_2410_08661_amd import binding as B
    san = C.CDLL(sys.argv[1])
    for name, (res, args) in B.EXPORTS.items():
        fn = getattr(san, name)
        fn.restype, fn.argtypes = res, args
    P, big, n = 0x100000, 2**31 - 1, 0
    def both(name, *args):
        global n
        n += 1
        a, b = getattr(B.raw, name)(*args), getattr(san, name)(*args)
        assert a == b, (name, a, b)
        return a
    for width, dtype, scale in itertools.product((-1, 0, 1, 7, 32000, 131073, 2**24, big), (0, 1, 2), (1.0, 0.0, float("nan"))):
        d = B.qeft_logprob_desc_t(width, dtype, scale)
        for m, top in itertools.product((-1, 0, 1, 57, 4096, 2**21, 2**21 + 1, 2**40, 2**63 - 1), (-1, 0, 1, 64, 65, big)):
            both("qeft_logprob_workspace", C.byref(d), m, top)
            f = B.qeft_logprob_fwd_t(P, P + 2, P, P, P, P, P, 2**40, 64, m, top, P, 2**40)
            b = B.qeft_logprob_bwd_t(P, P + 2, P, P, P, P, P, P, 2**40, 2**40, m)
            if m != 0:
                assert both("qeft_logprob_fwd", C.byref(d), C.byref(f), None) != 0
                assert both("qeft_logprob_bwd", C.byref(d), C.byref(b), None) != 0
                assert both("qeft_logprob_fwd_bwd", C.byref(d), C.byref(f), C.byref(b), None) != 0
    for hd, heads, kv, rot in itertools.product((-8, 0, 8, 40, 128, 256, 264, big), (-1, 0, 1, 64, 2**24, big), (0, 1, 2**24, big), (-2, 0, 2, 31, 256, big)):
        d = B.qeft_qk_desc_t(hd, heads, kv, rot, 1e-6)
        for m in (-1, 0, 1, 4001, 2**21, 2**21 + 1, 2**40):
            both("qeft_qk_norm_workspace", C.byref(d), m)
            if m != 0:
                f = B.qeft_qk_fwd_t(P, P, P + 2, P, P, P, P + 2, P, 2**40, 2**40, 2**40, 2**40, 2**40, m, 9)
                assert both("qeft_qk_norm_fwd", C.byref(d), C.byref(f), None) != 0
                g = B.qeft_qk_bwd_t(P, P, P, P, P + 2, P, P, P, P, 2 * P, P, P, 2**40, 2**40, 2**40, 2**40, 2**40, 2**40, 2**40, m, 9, 0, P, 2**40)
                assert both("qeft_qk_norm_bwd", C.byref(d), C.byref(g), None) != 0
    # lists: sizes at their limits, addresses at the end of the address space
    for sizes, at, bits in itertools.product(((1,), (0, 5), (8192, 8193, 1), (2**40,), (2**40 + 1,), (-1,), (2**40,) * 9, ()), (P, 2**47, 2**64 - 2**20), (8, 32, 4)):
        rows = (B.qeft_tensor_t * max(1, len(sizes)))()
        for i, s in enumerate(sizes):
            where = iter(range(7 * i, 7 * i + 7))
            for name in ("weight", "master", "grad", "m", "v", "m_scale", "v_scale"):
                k = next(where)
                setattr(rows[i], name, 0 if bits != 8 and name.endswith("scale") else (at + k * 2**16) % 2**64)
            rows[i].n, rows[i].decay = s, 0.1
        size = both("qeft_tensors_plan_bytes", rows, len(sizes))
        if size < 2**24:
            bufs = [C.create_string_buffer(size + 32) for _ in range(2)]
            outs = [B.qeft_tensors_t() for _ in range(2)]
            got = [lib.qeft_tensors_plan(rows, len(sizes), 1, bits, C.addressof(b) + 15 & ~15, size, C.byref(o)) for lib, b, o in zip((B.raw, san), bufs, outs)]
            assert got[0] == got[1] and bytes(outs[0]) == bytes(outs[1])
            data = [C.string_at(C.addressof(b) + 15 & ~15, size) for b in bufs]
            assert data[0] == data[1]
            n += 1
    for work, count, dt, bits in itertools.product((-1, 0, 1, 2**30, 2**30 + 1, 2**62), (-1, 0, 5, 2**20 + 1, big), (0, 1, 2), (8, 32, 33)):
        l = B.qeft_tensors_t(P, work, count, dt, bits, 1, 1)
        both("qeft_grad_norm_workspace", C.byref(l))
        if work != 0:
            for b1, step in itertools.product((0.0, 0.9, 1.0, -1.0), (-2**63, 0, 1, 2**30, 2**63 - 1)):
                a = B.qeft_adamw_t(0.1, b1, 0.999, 1e-8, step, 2**64 - 1, 0, 0, P + 2, 1)
                assert both("qeft_adamw_step", C.byref(l), C.byref(a), None) != 0
            g = B.qeft_grad_norm_t(1.0, 1.0, P + 2, 0, P, 2**40)
            assert both("qeft_grad_norm", C.byref(l), C.byref(g), None) != 0
    print("calls compared:", n)
''')


@pytest.mark.skipif(not os.path.exists(qbuild.HIPCC), reason="needs hipcc")
def test_host_logic_under_ubsan(tmp_path):
    objs = [os.path.join(qbuild.BUILD_DIR, f[:-4] + ".o") for f in qbuild.SOURCES if f[:-4] not in FILES]
    if not all(os.path.exists(o) for o in objs):
        pytest.skip("regular build objects are missing: run `python -m paper_2410_08661_amd.build` first")
    san = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [f for f in qbuild.FLAGS if f != "-O3"]
    jobs = [subprocess.Popen([qbuild.HIPCC, *flags, "-O1", *san, "-c", os.path.join(qbuild.CSRC, f + ".hip"), "-o", str(tmp_path / (f + ".o"))],
                             stdout=subprocess.DEVNULL, stderr=subprocess.PIPE) for f in FILES]
    for j in jobs:
        err = j.communicate()[1]
        assert j.returncode == 0, err.decode()[-2000:]
    rt_dirs = glob.glob(os.path.join(os.path.dirname(os.path.realpath(qbuild.HIPCC)), "..", "lib", "llvm", "lib", "clang", "*", "lib", "linux"))
    rt = [d for d in rt_dirs if os.path.exists(os.path.join(d, "libclang_rt.ubsan_standalone-x86_64.so"))]
    if not rt:
        pytest.skip("the toolchain ships no shared UBSan runtime")
    lib = str(tmp_path / "libqeft_ubsan.so")
    subprocess.run([qbuild.HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib, *(str(tmp_path / (f + ".o")) for f in FILES), *objs, "-L", rt[0],
                    "-l:libclang_rt.ubsan_standalone-x86_64.so", f"-Wl,-rpath,{os.path.realpath(rt[0])}"], check=True, capture_output=True)
    r = subprocess.run([sys.executable, "-c", CHILD, lib], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "runtime error" not in r.stderr, r.stderr[-3000:] + r.stdout[-500:]
    assert "calls compared:" in r.stdout
