"""Which kernels the head's products run on, on the host: csrc/matmul.hip and csrc/head_loss.hip compiled for the CPU with launches that write down
what they were asked for, over batches, widths and vocabularies."""
import os
import subprocess

import paper_2502_04416_amd

CSRC = os.path.join(os.path.dirname(paper_2502_04416_amd.__file__), "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

HEAD = r'''
#include "matmul.hip"
#include "head_loss.hip"
#include <cstdio>
#include <cstdlib>

namespace cmoe {
Tuning& tuning() { static Tuning t; return t; }
int fail(int code, const char*, ...) { return code; }
size_t elem_size(int dtype) { return dtype == CMOE_F32 ? 4 : 2; }
#define NOT_HERE(name) hipError_t name(Tile, int, const MatArgs&, hipStream_t) { return hipErrorInvalidValue; }
NOT_HERE(launch_gated) NOT_HERE(launch_dgated) NOT_HERE(launch_down) NOT_HERE(launch_dx) NOT_HERE(launch_dw) NOT_HERE(launch_lse) NOT_HERE(launch_dlogits) NOT_HERE(launch_dhead)
}  // namespace cmoe
using namespace cmoe;
'''


def run(tmp_path, name, body):
    src, exe = tmp_path / (name + ".cpp"), tmp_path / name
    src.write_text(HEAD + body)
    built = subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-O1", "-std=c++17", "-w", "-I" + CSRC,
                            str(src), "-o", str(exe)], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_all_pieces_of_a_vocabulary_have_one_order_of_sums(tmp_path):
    """Forward and backward pieces, the last ones a few entries wide too: the ring for all or the kernel for any operand for all, K split alike, and
    where that kernel runs, 16 bytes of every operand."""
    run(tmp_path, "pieces", r'''
int main() {
  long seen[2] = {0, 0};
  for (int dtype : {CMOE_BF16, CMOE_F32})
    for (int direct = 0; direct <= (dtype == CMOE_BF16); ++direct)
      for (long t : {1, 2, 7, 64, 65, 300, 2048, 65600, 262144})
        for (long d : {1, 2, 3, 5, 7, 8, 9, 12, 14, 15, 16, 24, 33, 64, 515, 1024, 4096, 40000})
          for (long v : {1, 2, 3, 7, 8, 9, 15, 40, 130, 1023, 1025, 2051, 4097, 4099, 8193, 32768, 131075}) {
            if (direct && d % 8) continue;
            const ForwardSpace f(dtype, t, d, v);
            const BackwardSpace b(dtype, t, d, v);
            int family = -1, split = -1;
            auto look = [&](const char* what, Product kind, long n, long n_b, size_t room) {
              const Choice c = choose(kind, dtype, direct, false, t, n, d, room, kind == PRODUCT_LSE ? &f.plan : &b.plan);
              const int ring = c.tile <= RING_64;
              if ((family >= 0 && ring != family) || (split >= 0 && c.k_split != split) || (!ring && (t * d < 8 || n_b * d < 8)) || (ring && !direct && !c.copies)) {
                printf("dtype %d direct %d, %ld tokens of %ld over %ld, %s of %ld: ring %d (%d), split %d (%d)\n", dtype, direct, t, d, v, what, n, ring, family, c.k_split, split);
                exit(1);
              }
              family = ring, split = c.k_split, ++seen[ring];
            };
            for (long n : {f.piece, f.last}) look("forward piece", PRODUCT_LSE, n, n, f.total - f.product);
            for (long n : {b.piece, v - (v - 1) / b.piece * b.piece}) look("backward piece", PRODUCT_DLOGITS, (n + 7) / 8 * 8, n, b.total - b.product);
          }
  return seen[0] > 500 && seen[1] > 500 ? 0 : 2;
}
''')
