"""The sum of row units' weights against walking through them, on the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "subgen_paged.cuh"

// as Plan's own_limit, unit_tiles and unit_weight say, one unit after the other
static long long walked(int units, int S, int nq, int prefix, int causal, int RU, int g, int KT, int lead) {
    long long w = 0;
    const long long rows = (long long)nq << g;
    for (int k = 0; k < units; ++k) {
        const long long last = std::min(rows, (k + 1LL) * RU) - 1;
        long long lim = causal ? S - nq + 1 + (last >> g) : S;
        lim = lim < 0 ? 0 : lim > S ? S : lim;
        const long long tiles = prefix + (lim + KT - 1) / KT;
        w += tiles ? lead + tiles : 0;
    }
    return w;
}

int main() {
    std::mt19937 r(1);
    auto up_to = [&](int n) { return (int)(r() % (unsigned)(n + 1)); };
    for (int i = 0; i < 20000; ++i) {
        const int rus = 3 + up_to(1), g = up_to(3), kt = 7, lead = 1 + up_to(3), causal = up_to(3) > 0;
        const int most = up_to(9) ? 300 : 20000, nq = up_to(most), S = up_to(3) ? up_to(most + 400) : nq + up_to(1), prefix = up_to(1) * up_to(5);
        const int all = (int)((((long long)nq << g) + (1 << rus) - 1) >> rus);
        for (int units : {0, 1, up_to(all), all - 1, all}) {
            if (units < 0 || units > all) continue;
            const long long a = sgk::first_units_weight(units, S, nq, prefix, causal, rus, g, kt, lead), b = walked(units, S, nq, prefix, causal, 1 << rus, g, 1 << kt, lead);
            if (a != b) { printf("units %d of %d, S %d, nq %d, prefix %d, causal %d, RU %d, g %d: %lld, not %lld\n", units, all, S, nq, prefix, causal, 1 << rus, g, a, b); return 1; }
        }
    }
    // the longest that a call takes: no sum overflows
    const int nq = 1 << 29, S = 0x7fffffff - 1024;
    const long long a = sgk::first_units_weight(1 << 26, S, nq, 100, 1, 3, 0, 7, 2), b = walked(1 << 26, S, nq, 100, 1, 8, 0, 128, 2);
    if (a != b) { printf("%lld, not %lld\n", a, b); return 1; }
    puts("ok");
}
"""


def test_units_are_summed_up_as_they_are_walked(tmp_path):
    src, exe = tmp_path / "plan.cu", str(tmp_path / "plan")
    src.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2402_06082_b200", "csrc"),
                           "-o", exe, str(src)])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout
