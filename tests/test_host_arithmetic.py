"""Host code of the library built without optimisation, where nothing that is computed and not used drops out: calls that have
nothing to sum have to get as far as the launch."""
import os
import subprocess

from paper_2605_01989_b200 import build as lib_build

PROGRAM = r"""
#include <stdarg.h>
#include <stdio.h>
#include "norm_rotate.cu"

namespace dblp {
std::atomic<uint64_t> g_launches{0};
void set_error(const char*, ...) {}
}  // namespace dblp

int main()
{
    alignas(256) static char ws[1 << 20];
    static float dw[64];
    const uint32_t shapes[3][2] = {{2, 0}, {0, 5}, {0, 0}};
    for (auto& s : shapes) {
        dblp_norm_rotate_t a{};
        a.batch = s[0];
        a.tokens = s[1];
        a.q_heads = a.k_heads = 3;
        a.head_dim = 64;
        a.eps = 1e-6f;
        printf("%d\n", dblp_norm_rotate_grad(&a, nullptr, nullptr, nullptr, nullptr, dw, nullptr, nullptr, nullptr, nullptr, nullptr, ws, sizeof ws, nullptr));
    }
}
"""


def test_a_gradient_of_no_tokens_divides_by_nothing(tmp_path):
    source, program = tmp_path / "no_tokens.cu", tmp_path / "no_tokens"
    source.write_text(PROGRAM)
    subprocess.run([lib_build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xptxas", "-O0", "-I",
                    os.path.join(lib_build.ROOT, "include"), "-I", lib_build.CSRC, "-o", program, source], check=True)
    # without a device the launch is where the call ends; the addresses are the host's
    run = subprocess.run([program], env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, capture_output=True, text=True)
    assert run.returncode == 0, run.returncode
    assert run.stdout.split() == ["-4"] * 3
