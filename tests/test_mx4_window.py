"""The loads of the packed microscaled weight that run ahead of the product, held against the weight's end on the host.  No GPU."""
import os
import subprocess

from paper_2509_09090_amd import build

PROGRAM = """
#include <cstdio>
#include <hip/hip_runtime.h>
#include "mx4_stage.h"

// a wavefront's fragments, its stages in flight and the stages of K: every load that the kernel makes for a stage that there is or that lies ahead
int main()
{
    int wrong = 0, loads = 0;
    for (int fragments = 1; fragments <= 2; ++fragments)
        for (int depth = 1; depth <= 4; ++depth)
            for (int stages = 1; stages <= 4096; stages += stages < 40 ? 1 : 1014)
                for (int c = 0; c < fragments; ++c)
                    for (int st = 0; st < stages + depth; ++st, ++loads) {
                        const unsigned long long codes = sqap::weight_stage(c, st, stages, 4096u), scales = sqap::weight_stage(c, st, stages, 256u);
                        // (three fragments of 1 KiB and 63 lanes of 16 bytes on; 63 lanes of 4)
                        wrong += codes + 3 * 1024 + 63 * 16 + 16 > 4096ull * stages * fragments;
                        wrong += scales + 63 * 4 + 4 > 256ull * stages * fragments;
                        wrong += st < stages && (codes != 4096ull * (c * stages + st) || scales != 256ull * (c * stages + st));
                    }
    std::printf("%d loads, %d outside\\n", loads, wrong);
    return wrong != 0 || loads == 0;
}
"""


def test_loads_ahead_stay_inside_the_weight(tmp_path):
    source, program = tmp_path / "window.hip", tmp_path / "window"
    source.write_text(PROGRAM)
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-I", os.path.join(build.HERE, "csrc"), str(source), "-o", str(program)],
                   check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
