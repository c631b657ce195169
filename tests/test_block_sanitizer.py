"""The host side of the calls between the linear layers (argument checks, plans and workspace sizes up to the first HIP call) rebuilt with the undefined-behaviour
sanitizer and swept through the C ABI without a GPU, every answer compared with the regular library's."""
import glob
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2410_08661_amd import build as qbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ["block_api", "append", "attn", "evict", "norm"]

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
    sizes = [-1, 0, 1, 7, 64, 511, 513, 4096, 131072, 2**24, 2**24 + 1, 2**40]
    for pages, page, kv, d in itertools.product((0, 1, 5000, big), (0, 1, 7, 16, 2**24, big), (1, 8, 40, 2**22, big), (0, 8, 60, 128, 256, 264)):
        desc = B.make_cache_desc(pages, page, kv, d, 4096, 512, d)
        for seqs, longest in itertools.product((-1, 0, 1, 8, 300, 2**24, 2**40), sizes):
            for heads in (0, kv, 8 * kv if kv < 2**27 else big):
                for w in (0, 1):
                    both("qeft_attn_workspace", C.byref(desc), seqs, min(heads, big), longest, w)
            for budget in (-1, 0, 1, 100, 4096, 2**24, 2**40):
                both("qeft_evict_workspace", C.byref(desc), seqs, longest, budget)
    for width, gate, res in itertools.product((-1, 0, 1, 4096, 8193, 16385, 2**24, big), (-1, 0, 1, 2, 3), (0, 1, 2)):
        desc = B.qeft_norm_desc_t(width, res, gate, 1.0, 1e-5)
        for m in (-1, 0, 1, 333, 4096, 2**21, 2**21 + 1, 2**40):
            both("qeft_norm_workspace", C.byref(desc), m)
    # refusals: every call below must return before a launch
    desc, pools = B.make_cache_desc(8, 16, 4, 64), B.qeft_cache_t(P, P)
    for seqs, cols, ld in itertools.product((-1, 1, 2**24, big), (-1, 0, 4, big), (0, 4, 2**40)):
        table = B.qeft_table_t(P, ld, cols, seqs)
        for longest in (-1, 64, 2**24, 2**40):
            attn = B.qeft_attn_t(P + 2, longest, P, P, 512, 512, 8, 1.0, P, longest, 0, 0, 0)     # misaligned lengths
            assert both("qeft_attn_decode", C.byref(desc), C.byref(pools), C.byref(table), C.byref(attn), None) != 0
            ev = B.qeft_evict_t(P + 2, P, longest, longest // 2, P, 2 * P, 2**40, 0, 0, 3 * P, 4 * P, 2**40, 5 * P, 0, 0)
            assert both("qeft_cache_evict", C.byref(desc), C.byref(pools), C.byref(table), C.byref(ev), None) != 0
            ap = B.qeft_append_t(P, P, P, P, 512, 512, 256, 256, P, P + 2, P, P, 64, 9, 64, 8, longest)
            assert both("qeft_cache_append", C.byref(desc), C.byref(pools), C.byref(table), C.byref(ap), None) != 0
    for m in (-1, 1, 2**21, 2**40):
        nd = B.make_norm_desc(64, gate=B.QEFT_GATE_TOKEN)
        fw = B.qeft_norm_fwd_t(P, P, P, P, P + 2, P, P, 64, 64, 2**40, 64, 64, m)
        assert both("qeft_norm_fwd", C.byref(nd), C.byref(fw), None) != 0
        bw = B.qeft_norm_bwd_t(P, P, P, P, P, P, P, P, P, P, P, P, 64, 64, 64, 64, 64, 64, 64, 64, m, 0, P + 4, 2**40)
        assert both("qeft_norm_bwd", C.byref(nd), C.byref(bw), None) != 0
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
