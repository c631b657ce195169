"""Dynamic LDS beyond what a launch gets by default has to be allowed for a kernel on each device.  A host program takes the HIP runtime's place under the library (its
launches do nothing), sweeps the entry points on one device and then on another, and counts launches of much LDS whose kernel has no such allowance on the
device that is current."""
import os
import shutil
import subprocess

import pytest

from paper_2410_08661_amd import build as qbuild

PROGRAM = r'''
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <map>
#include <set>
#include <string>
#include <utility>
#include "qeft.h"

struct dim3 { uint32_t x, y, z; };
static int device = 0, refuse = 0;
static long launches = 0, missing = 0;
static std::map<std::pair<int, const void*>, size_t> allowed;
static std::map<const void*, std::string> names;
static std::set<std::string> large[2];
static struct { dim3 g, b; size_t lds; void* s; } pushed;

extern "C" {   // what libqeft takes from the HIP runtime
void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names[f] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, void* s) { pushed = {g, b, lds, s}; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, void** s) { *g = pushed.g, *b = pushed.b, *lds = pushed.lds, *s = pushed.s; return 0; }
int hipGetDevice(int* d) { *d = device; return 0; }
int hipGetLastError() { return 0; }
int hipGetSymbolAddress(void** p, const void*) { *p = (void*)0x7000000; return 0; }
int hipFuncSetAttribute(const void* f, int, int bytes) {
    if (refuse) return 1;
    size_t& most = allowed[{device, f}];
    if ((size_t)bytes > most) most = bytes;
    return 0;
}
int hipLaunchKernel(const void* f, dim3, dim3, void**, size_t lds, void*) {
    ++launches;
    if (lds <= 60 * 1024) return 0;
    large[device].insert(names[f]);
    const auto it = allowed.find({device, f});
    if (it == allowed.end() || it->second < lds) {
        if (++missing <= 5) printf("device %d, %zu bytes: %s\n", device, lds, names[f].c_str());
    }
    return 0;
}
}

int main(int, char** argv) {
    void* lib = dlopen(argv[1], RTLD_NOW);
    if (!lib) { printf("%s\n", dlerror()); return 2; }
#define F(name) const auto name##_ = (decltype(&name))dlsym(lib, #name)
    F(qeft_linear_fwd); F(qeft_linear_bwd_dx); F(qeft_linear_bwd); F(qeft_weak_grad); F(qeft_linear_fwd_irregular); F(qeft_workspace_bytes);
    F(qeft_cache_evict); F(qeft_evict_workspace); F(qeft_norm_bwd); F(qeft_norm_workspace);
    char* P = (char*)0x100000;          // addresses that nothing reads
    char* ws = (char*)0x40000000;
    const size_t much = (size_t)1 << 40;
    auto sweep = [&] {
        const int sizes[][2] = {{512, 512}, {4096, 4096}, {11008, 4096}, {4096, 11008}, {8192, 28672}, {5120, 5120}, {4104, 4104}, {1024, 40960}};
        for (auto& sz : sizes)
            for (int k : {8, 64, 128, 256, 129})
                for (int bits : {43, 4, 3, 30})
                    for (int g : {128, 64}) {
                        qeft_desc_t d{sz[0], sz[1], k, bits == 43 ? 4 : bits == 30 ? 3 : bits, g, bits == 30 ? QEFT_LAYOUT_DENSE3 : QEFT_LAYOUT_CANONICAL};
                        qeft_weight_t w{P, P, P, P};
                        for (int64_t M : {1, 2, 4, 8, 16, 17, 32, 64, 100, 192, 300, 512, 1000, 2048, 4096})
                            for (size_t n : {(size_t)0, much}) {
                                void* p = n ? ws : nullptr;
                                const int64_t kw = k > 8 ? (k + 7) / 8 * 8 : 8;
                                qeft_linear_fwd_(&d, &w, P, M, sz[1], P, sz[0], p, n, nullptr);
                                qeft_linear_fwd_irregular_(&d, &w, (int32_t*)P, P, M, sz[1], P, sz[0], p, n, nullptr);
                                qeft_linear_bwd_dx_(&d, &w, P, M, sz[0], P, sz[1], p, n, nullptr);
                                qeft_weak_grad_(&d, P, M, sz[0], P, kw, P, QEFT_DTYPE_F32, 0, p, n, nullptr);
                                qeft_linear_bwd_(&d, &w, P, M, sz[0], P, sz[1], P, kw, P, QEFT_DTYPE_F32, 0, p, n, nullptr);
                            }
                    }
        const qeft_cache_desc_t cd{4096, 16, 4, 64, 4096, 1024, 64};
        const qeft_cache_t pools{P, P};
        for (int64_t longest : {100, 4000, 8000, 16000, 20000, 32768, 40000})
            for (int64_t ld : {longest, longest + 1}) {
                const qeft_table_t t{(int32_t*)P, 4096, 4096, 2};
                float* s = (float*)(P + (1 << 24));
                qeft_evict_t e{(int32_t*)P, (int32_t*)(P + 4096), longest, longest / 2, s, (int32_t*)(P + (1 << 25)), ld, 0, 0, s, (int32_t*)(P + (1 << 25)), ld, (int32_t*)(P + 8192), ws, much};
                const int st = qeft_cache_evict_(&cd, &pools, &t, &e, nullptr);
                if (st) printf("evict %ld: %d\n", (long)longest, st), ++missing;
            }
        for (int n : {512, 4096, 8192, 12000, 16384, 20000})
            for (int res : {0, 1})
                for (int gate : {0, 1, 2})
                    for (bool post : {false, true}) {
                        const qeft_norm_desc_t d{n, res, gate, 1.f, 1e-5f};
                        void* g = gate ? P : nullptr;
                        qeft_norm_bwd_t b{P, P, P, P, g, P, post ? P : nullptr, P, P, g, (float*)P, post ? (float*)P : nullptr, n, n, n, n, n, n, n, n, 300, 0, ws, much};
                        const int st = qeft_norm_bwd_(&d, &b, nullptr);
                        if (st) printf("norm %d: %d\n", n, st), ++missing;
                    }
    };
    for (int d : {0, 1, 0}) {
        device = d;
        sweep();
    }
    printf("launches %ld, kernels of much LDS %zu and %zu, not allowed %ld\n", launches, large[0].size(), large[1].size(), missing);
    // an allowance that the runtime refuses is the call's error
    device = 1, refuse = 1;
    const qeft_norm_desc_t d{16384, 1, 0, 1.f, 1e-5f};
    qeft_norm_bwd_t b{P, P, P, P, nullptr, P, P, P, P, nullptr, (float*)P, (float*)P, 16384, 16384, 16384, 16384, 0, 16384, 16384, 0, 300, 0, ws, much};
    const long before = launches;
    const int st = qeft_norm_bwd_(&d, &b, nullptr);
    printf("refused: %d, launches after it %ld\n", st, launches - before);
    return missing != 0 || large[0] != large[1] || large[0].size() < 20 || st != QEFT_ERR_HIP || launches != before;
}
'''


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_device_allows_what_is_launched_on_it(tmp_path):
    if not os.path.exists(qbuild.LIB_PATH):
        pytest.skip("the library is not built")
    src, exe = tmp_path / "sweep.cpp", tmp_path / "sweep"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(qbuild.ROOT, "include"), str(src), "-o", str(exe), "-ldl"], check=True)
    r = subprocess.run([str(exe), qbuild.LIB_PATH], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]
