"""Products whose 8-bit operands no kernel of the call would read are refused:
a small host program against the built library makes the internal calls (no
device code is compiled and nothing is launched)."""
import os
import subprocess

import pytest

from paper_2507_03312_amd import build as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB) or not os.path.exists(B.HIPCC),
                                reason="libmpx.so or hipcc missing")

SOURCE = r"""
#include <cstdio>
#include <cstring>
#include "gemm_kernels.h"
using namespace mpx;
static char at[64] __attribute__((aligned(64)));  // never dereferenced
static GemmArgs product(int64_t M, int64_t N, int64_t K, bool ak, bool bk) {
  GemmArgs g{};
  g.nb1 = 1;
  g.splits = 1;
  g.M = M; g.N = N; g.K = K;
  g.A = (const uint16_t*)at; g.B = (const uint16_t*)at; g.C = (uint16_t*)at;
  g.lda = ak ? K : M; g.ldb = bk ? K : N; g.ldc = N;
  return g;
}
int main(int argc, char** argv) {
  const char* what = argv[1];
  const bool f16 = !strcmp(argv[2], "f16");
  const auto is = [&](const char* s) { return !strcmp(what, s); };
  bool ak = true, bk = false;
  if (is("forward")) bk = true;
  if (is("weight gradient") || is("its 8-bit form")) ak = false;
  // direct tiles, register-staged ones, ones of any operands
  const int64_t sizes[3][3] = {{256, 256, 128}, {257, 131, 65}, {129, 5, 40}};
  int64_t nbatch = 1;
  for (const auto& z : sizes) {
    GemmArgs g = product(z[0], z[1], z[2], ak, bk);
    g.dact8 = g.dact8_scale = (const uint8_t*)at;
    if (is("count")) g.nonfinite = (int32_t*)at;
    if (is("bias")) g.bias = (const uint16_t*)at;
    if (is("residual")) { g.resid = (const uint16_t*)at; g.ldr = g.N; }
    if (is("gelu")) { g.act = MPX_ACT_GELU_TANH; g.pre = (uint16_t*)at; }
    if (is("both pre-activations")) g.dact = (const uint16_t*)at;
    if (is("splits")) { g.splits = 2; g.k_split = 64; g.ws = (float*)at; }
    if (is("batch")) nbatch = 2;
    if (is("no scales")) g.dact8_scale = nullptr;
    if (is("8-bit B")) { g.dact8 = g.dact8_scale = nullptr; g.b8 = g.b8_scale = (const uint8_t*)at; }
    if (is("half B")) g.dact8 = g.dact8_scale = nullptr;
    hipError_t e;
    bool fused = false;
    if (is("its 8-bit form") || is("half B")) {
      if (is("its 8-bit form")) g.b8 = g.b8_scale = (const uint8_t*)at;
      e = f16 ? run_gemm_act8_f16(g, nullptr, &fused) : run_gemm_act8_bf16(g, nullptr, &fused);
    } else {
      e = f16 ? run_gemm_f16(g, ak, bk, nbatch, nullptr, &fused) : run_gemm_bf16(g, ak, bk, nbatch, nullptr, &fused);
    }
    if (e != hipErrorInvalidValue) {
      printf("%s: %lld x %lld x %lld gave %d\n", what, (long long)g.M, (long long)g.N, (long long)g.K, (int)e);
      return 1;
    }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("gemm_operands")
    src, exe = str(d / "main.hip"), str(d / "main")
    with open(src, "w") as f:
        f.write(SOURCE)
    flags = [f for f in B.FLAGS if f not in ("-O3", "--offload-arch=gfx950")]
    cmd = [B.HIPCC, "--offload-host-only", "-O0", *flags, src, "-o", exe, "-L", B.PKG, "-l:libmpx.so",
           f"-Wl,-rpath,{B.PKG}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return exe


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("what", ["count", "bias", "residual", "gelu", "both pre-activations", "splits", "batch",
                                  "forward", "weight gradient", "its 8-bit form", "no scales", "8-bit B", "half B"])
def test_refused(program, what, fmt):
    env = {**os.environ, "HIP_VISIBLE_DEVICES": "-1"}
    r = subprocess.run([program, what, fmt], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
