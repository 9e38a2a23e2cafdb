"""How the products of the orthogonalising iteration are cut for given matrices: the host's own code of
csrc/train_api.cu, compiled into a small program that prints its plans."""
import functools
import os
import subprocess
import tempfile

from paper_2603_06492_gb300.build import ARCH, CSRC

MAIN = r"""
}  // namespace
}  // namespace noble

// rows cols ...; prints "group phase unit-total" and "matrix phase tile-columns tiles-of-rows splits pieces" lines
int main(int argc, char **argv)
{
    using namespace noble;
    std::vector<noble_muon_tensor> t;
    for (int i = 2; i + 1 < argc; i += 2) {
        noble_muon_tensor m{};
        m.rows = atoll(argv[i]), m.cols = atoll(argv[i + 1]);
        t.push_back(m);
    }
    for (int next = 0; next < (int)t.size();) {
        const MuonPlan w = muon_plan(t.data(), (int)t.size(), &next, (uint32_t)atoi(argv[1]));
        for (int j = 0; j < kPhases && !w.small; ++j) {
            printf("G %d %d %d\n", w.n, j, w.units[j]);
            for (int i = 0; i < w.n; ++i) {
                const muon::mma::Problem &p = w.p[j][i];
                printf("P %d %d %d %d %d %d %d %d\n", w.pick[i], j, p.bn, p.tiles_m, p.tiles_n, p.nsplit,
                       (p.kb_per_split + p.piece_kb - 1) / p.piece_kb, p.segs);
            }
        }
    }
}
"""


@functools.lru_cache
def _program():
    with open(os.path.join(CSRC, "train_api.cu")) as f:
        text = f.read()
    # from the rule on pairs to the last line of the plan
    start, end = text.index("// Small matrices cost launches"), text.index("// TMA map of an fp16 matrix")
    head = '#include <algorithm>\n#include <cstdlib>\n#include "host.cuh"\n#include "muon_small.cuh"\nnamespace noble {\nnamespace {\n'
    work = tempfile.mkdtemp(prefix="muon_plan")
    src, exe = os.path.join(work, "plan.cu"), os.path.join(work, "plan")
    with open(src, "w") as f:
        f.write(head + text[start:end] + MAIN)
    subprocess.run([os.environ.get("NVCC", "nvcc"), *ARCH, "-O1", "-std=c++17", "-I" + CSRC, src, "-o", exe], check=True,
                   capture_output=True)
    return exe


GRAM, POLY, NEXT = range(3)  # X X^T, the polynomial of A, B X


def plan(shapes, flags=0):
    """[(units of the group's launch, phase, [dict of each matrix])] of every launch of a step."""
    out = subprocess.run([_program(), str(flags), *(str(n) for s in shapes for n in s)], check=True, capture_output=True, text=True)
    launches = []
    for line in out.stdout.splitlines():
        kind, *v = line.split()
        v = [int(x) for x in v]
        if kind == "G":
            launches.append((v[2], v[1], []))
        else:
            launches[-1][2].append(dict(zip(("matrix", "phase", "bn", "tiles_m", "tiles_n", "nsplit", "pieces", "segs"), v)))
    return launches
