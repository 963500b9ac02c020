"""Which kernels the calls of layer norm, the point-wise product and dropout launch, and how large, asked of the library's own host code by a small
program that notes its launches in place of making them."""
import os
import subprocess

from tests.test_abi_host import ROOT

HIPCC = "/opt/rocm/bin/hipcc"
CSRC = os.path.join(ROOT, "paper_2503_06671_amd", "csrc")
SOURCES = ("esc_norm.hip", "esc_product.hip", "esc_product_strip.hip", "esc_dropout.hip")

NOTED = r"""
#pragma once
#include <hip/hip_runtime.h>
void launched(const void *kernel, dim3 grid, dim3 block);
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, ...) launched((const void *)(kernel), grid, block)
#define hipGetLastError() hipSuccess
#define hipFuncSetAttribute(...) hipSuccess
"""

PROGRAM = r"""
#include <stdio.h>
#include <hip/hip_runtime.h>
#include <map>
#include <string>
#include "esc_convattn.h"
// (the kernels themselves are not built into this program; what registers them gives their names)
static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}
void launched(const void *kernel, dim3 grid, dim3 block)
{
    printf("launch %lu %u %u %u %s\n", (unsigned long)grid.x, grid.y, grid.z, block.x, names().at(kernel).c_str());
}
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *none; return &none; }
void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned, void *, void *, void *, void *, int *) { names()[host] = device; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void **) {}
}
// lines in: call dt N K M H W act flag; the launches, then the status, out.  flag: a residual; of the product's gradients 1: not x's, 2: not w's
static void *at(unsigned long i) { return (void *)(i << 59); }   // no memory, and none is touched
int main()
{
    int call, dt, N, K, M, H, W, act, flag;
    while (scanf("%d %d %d %d %d %d %d %d %d", &call, &dt, &N, &K, &M, &H, &W, &act, &flag) == 9) {
        const long P = (long)H * W;
        int st = -1;
        if (call < 2) {
            esc_layernorm a{N, K, H, W, 1e-5f, (const float *)at(1), (const float *)at(2), K * P, K * P, K * P};
            esc_layernorm_grads g{at(5), K * P, (float *)at(6), (float *)at(7)};
            st = call == 0 ? esc_layernorm_forward(at(3), (esc_dtype)dt, &a, at(4), at(8), (size_t)-1 / 4, nullptr)
                           : esc_layernorm_backward(at(3), at(4), nullptr, (esc_dtype)dt, &a, at(8), (size_t)-1 / 4, &g, 0, at(9), (size_t)-1 / 4, nullptr);
        } else if (call < 4) {
            esc_pointwise a{N, K, M, H, W, (esc_activation)act, (const float *)at(1), (const float *)at(2), K * P, M * P, M * P};
            esc_pointwise_grads g{at(5), K * P, (float *)at(6), (float *)at(7)};
            if (flag == 1) g.x = nullptr;
            if (flag == 2) g.w = nullptr;
            st = call == 2 ? esc_pointwise_forward(at(3), flag ? at(8) : nullptr, (esc_dtype)dt, &a, at(4), nullptr)
                           : esc_pointwise_backward(at(3), at(4), (esc_dtype)dt, &a, &g, 0, at(9), (size_t)-1 / 4, nullptr);
        } else {
            esc_dropout a{N, K, H, W, 0.25, (esc_dropout_over)act, 1, 2, nullptr, K * P, K * P, K * P};
            st = esc_dropout_forward(at(3), flag ? at(8) : nullptr, (esc_dtype)dt, &a, at(4), nullptr);
        }
        printf("status %d\n", st);
    }
}
"""

CALLS = {"layernorm_forward": 0, "layernorm_backward": 1, "pointwise_forward": 2, "pointwise_backward": 3, "dropout_forward": 4}


def build(at):
    """Compiles the program into the folder `at`; None where there is no compiler."""
    if not os.path.exists(HIPCC):
        return None
    (at / "noted.h").write_text(NOTED)
    (at / "main.cpp").write_text(PROGRAM)
    flags = [HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    jobs = []
    for s in SOURCES:
        jobs.append((at / f"{s}.o", subprocess.Popen([*flags, "-x", "hip", "-include", str(at / "noted.h"), "-c", os.path.join(CSRC, s), "-o", str(at / f"{s}.o")])))
    jobs.append((at / "main.o", subprocess.Popen([*flags, "-x", "hip", "-c", str(at / "main.cpp"), "-o", str(at / "main.o")])))
    assert all(p.wait() == 0 for _, p in jobs)
    subprocess.run([HIPCC, *(str(o) for o, _ in jobs), "-Wl,--unresolved-symbols=ignore-all", "-o", str(at / "launches")], check=True)
    return at / "launches"


class Launch:
    """grid and block, and the kernel's mangled name."""

    def __init__(self, line):
        *numbers, self.kernel = line.split()[1:]
        self.gx, self.gy, self.gz, self.block = (int(v) for v in numbers)

    def __repr__(self):
        return f"{self.kernel} grid {self.gx} x {self.gy} x {self.gz} of {self.block}"


def ask(program, calls):
    """calls: (name, dt, N, K, M, H, W, act, flag) each; a list of (status, [Launch, ...])."""
    text = "\n".join(" ".join(str(int(v)) for v in (CALLS[c[0]], *c[1:])) for c in calls)
    out = subprocess.run([str(program)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    res, held = [], []
    for line in out:
        if line.startswith("launch"):
            held.append(Launch(line))
        else:
            res.append((int(line.split()[1]), held))
            held = []
    assert len(res) == len(calls)
    return res
