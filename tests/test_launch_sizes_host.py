"""CPU test of the launches around a block's attention (compiled from the library's sources, with a recorder in the place of the
launch): whatever descriptor is accepted, no launch has 2^32 threads in a dimension or more than a grid takes, and the embedding's gradient
of few tokens goes the general way exactly where its one launch would have."""
import os
import shutil
import subprocess

import pytest

from paper_2501_08453_amd import build as B

HEAD = r"""
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdio>
#include <random>
#undef hipLaunchKernelGGL
static long launches, bad;
static void record(dim3 g, dim3 b) {
  ++launches;
  const uint64_t x = (uint64_t)g.x * b.x, y = (uint64_t)g.y * b.y;
  const bool ok = g.x >= 1 && g.y >= 1 && b.x >= 1 && b.y >= 1 && b.x * b.y <= 1024 && x < (uint64_t)1 << 32 && y < (uint64_t)1 << 32 && g.y < 65536;
  if (!ok && bad++ < 10) printf("grid %u x %u of %u x %u threads\n", g.x, g.y, b.x, b.y);
}
#define hipLaunchKernelGGL(kernel, grid, block, ...) record(grid, block)
#include "api_blocks.hip"
static std::mt19937_64 rng(7);
static int64_t spread(int64_t lo, int64_t hi) {  // over the logarithm, both ends among them
  const double u = std::uniform_real_distribution<double>(-0.05, 1.05)(rng);
  return u <= 0 ? lo : u >= 1 ? hi : std::min(hi, (int64_t)(lo * pow((double)hi / lo, u)));
}
"""

EMBEDDING = HEAD + r"""
#include "embedding.hip"
static long run(vc_embedding_desc d) {
  vcja::EmbeddingArgs a = embedding_args(&d, nullptr);
  a.dout_stride = a.table_stride = d.cols;
  a.out_f32 = d.out_type, a.grad_f32 = a.table_f32 = d.table_type, a.add = d.accumulate;
  const long before = launches;
  (void)vcja::launch_embedding_bwd(a, nullptr);
  return launches - before;
}
int main() {
  long few = 0, general = 0, wide = 0;
  for (int i = 0; i < 200000; ++i) {
    vc_embedding_desc d{spread(1, (rng() & 1) ? 64 : 1 << 24), spread(1, (int64_t)1 << 27), -1, 0, (int)spread(1, 8192), 1, (int)(rng() & 1),
                        (int)(rng() & 1), 1.0f, (int)(rng() & 1)};
    if (check_embedding(&d, true) != VC_OK) return 2;
    const long n = run(d);
    (n == 1 ? few : general) += 1;
    if (d.tokens > 64 && n < 2) return 3;
    if (d.accumulate && d.tokens <= 64 && n != 1) return 4;  // a launch of the tokens alone
    wide += d.tokens <= 64 && n > 1;
    vcja::EmbeddingArgs f = embedding_args(&d, nullptr);
    f.tokens = spread(1, 1 << 30);
    (void)vcja::launch_embedding_fwd(f, nullptr);
  }
  // 8,192 columns in bf16: four rows a workgroup of 1,024 threads; 2^22 workgroups would be 2^32 threads
  const int64_t most = 4 * (((int64_t)1 << 22) - 64 - 1);
  for (int64_t v : {most, most + 1}) {
    const long n = run(vc_embedding_desc{64, v, -1, 0, 8192, 1, 0, 0, 1.0f, 0});
    if ((n == 1) != (v == most)) return printf("%ld launches for a table of %ld rows\n", n, (long)v), 5;
  }
  printf("%ld of one launch, %ld of more, %ld of few tokens among these, %ld wrong\n", few, general, wide, bad);
  return bad ? 1 : few > 1000 && general > 1000 && wide > 10 ? 0 : 6;
}
"""

RESIDUAL = HEAD + r"""
#include "residual.hip"
int main() {
  long done = 0, shared = 0;
  for (int i = 0; i < 200000; ++i) {
    vc_residualnorm_desc d{};
    d.rows = spread(1, 1 << 30), d.cols = (int)spread(1, 8192), d.samples = (int)spread(1, 1 << 25);
    d.x_type = rng() & 1, d.y_type = d.x_type & (rng() & 1), d.norm = rng() % 3, d.post_norm = rng() % 3, d.packed = 1, d.residual_scale = 1.0f;
    if (check_residual(&d) != VC_OK) continue;
    ++done;
    (void)vcja::launch_residual_fwd(residual_args(&d, false), nullptr);
    vcja::ResidualArgs a = residual_args(&d, true);
    static float some;
    a.part = (rng() & 7) ? &some : nullptr;
    a.flat = d.samples == 1 || (rng() & 3) == 0;
    a.sums = a.part && !a.flat && (rng() & 1) ? &some : nullptr;
    shared += a.sums != nullptr;
    (void)vcja::launch_residual_bwd(a, rng() & 1, nullptr);
  }
  printf("%ld descriptors, %ld with sums over samples, %ld wrong\n", done, shared, bad);
  return bad ? 1 : done > 1000 && shared > 1000 ? 0 : 6;
}
"""

CHECKPOINT = HEAD + r"""
#include "checkpoint.hip"
int main() {
  for (int i = 0; i < 200000; ++i) {
    vc_checkpoint_desc d{spread(1, (int64_t)1 << 32), (int)spread(1, 1 << 24), (int)(rng() & 1), 0};
    if (check_checkpoint(&d) != VC_OK) return 2;
    const vcja::CheckpointArgs a = checkpoint_args(&d);
    (void)vcja::launch_checkpoint_pack(a, nullptr);
    (void)vcja::launch_checkpoint_unpack(a, nullptr);
  }
  printf("%ld launches, %ld wrong\n", launches, bad);
  return bad ? 1 : 0;
}
"""


@pytest.mark.parametrize("source", [EMBEDDING, RESIDUAL, CHECKPOINT], ids=["embedding", "residual", "checkpoint"])
def test_launches(tmp_path, source):
    try:
        cc = B.hipcc()
    except Exception as e:  # pragma: no cover - toolchain missing
        pytest.skip("hipcc not available: %s" % e)
    if not shutil.which(cc) and not os.path.exists(cc):
        pytest.skip("hipcc not available")
    src, exe = tmp_path / "sizes.hip", tmp_path / "sizes"
    src.write_text(source)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC", "-O3")]
    r = subprocess.run([cc, *flags, "-O1", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, str(src), "-o", str(exe), "-L" + B.PKG,
                        "-l:" + os.path.basename(B.LIB), "-Wl,-rpath," + B.PKG], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:])
