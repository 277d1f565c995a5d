"""Operators on ragged batches and 8-bit pages, without a device: what their sources promise, and sizes at the ends of their ranges."""
import glob
import os
import re
import subprocess

import paper_2403_09054_b200 as kf

CSRC = os.path.join(os.path.dirname(os.path.abspath(kf.__file__)), "csrc")


def _kernels():
    """(file, name, body) of the kernels of files that launch kernels before the one in front of them has ended."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = open(path).read()
        if "launch_early(" not in text:
            continue
        starts = [(m.start(), m.group(1)) for m in re.finditer(r"__global__ void __launch_bounds__\([^\n]*?\) (\w+)\(", text)]
        for (at, name), end in zip(starts, [s for s, _ in starts[1:]] + [len(text)]):
            yield os.path.basename(path), name, text[at:end]


def test_kernels_that_launch_early_wait_before_they_take_anything_that_lasts():
    """A kernel that holds tensor memory while it waits for the one before could keep that one from ever getting its own; and nothing of global memory may be touched."""
    seen = 0
    for file, name, body in _kernels():
        seen += 1
        wait = body.find("after_earlier_kernels();")
        assert wait >= 0, (file, name)
        for taken in ("tmem_alloc(", "P.begin[", "a.length[", "U.length[", "U.parent", "let_next_kernel_launch();"):
            at = body.find(taken)
            assert at < 0 or at > wait, (file, name, taken)
    assert seen >= 8


def test_scratch_of_sizes_beyond_32_bits():
    """What does not fit the argument structs is not supported: no bytes, not those of another size."""
    attend = dict(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_heads=4, n_kv_heads=2, head_dim=64)
    update = dict(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_kv_heads=2, head_dim=64, n_layers=2)
    assert kf.kf_pages_attend_scratch_bytes(**attend) > 0 and kf.kf_pages_update_scratch_bytes(**update) > 0
    for f, base in ((kf.kf_pages_attend_scratch_bytes, attend), (kf.kf_pages_update_scratch_bytes, update)):
        for name, value in base.items():
            for far in (value + 2 ** 32, value - 2 ** 32, 2 ** 31, 2 ** 70):
                assert f(**{**base, name: far}) == 0, (name, far)


HARNESS = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include "kf_args.cuh"
using namespace kf::args;
struct T { long at, a, sa, b, sb; int d; };
static std::set<long> bytes_of(const T& t) {
  std::set<long> s;
  for (long i = 0; i < t.a; ++i)
    for (long j = 0; j < t.b; ++j)
      for (long e = 0; e < 2 * t.d; ++e) s.insert(t.at + 2 * (i * t.sa + j * t.sb) + e);
  return s;
}
int main() {
  srand(1);
  long missed = 0, refused = 0, taken = 0;
  for (int n = 0; n < 60000; ++n) {
    T x{}, y{};
    x.d = 8 * (1 + rand() % 2); y.d = rand() % 2 ? x.d : 8 * (1 + rand() % 2);
    x.a = 1 + rand() % 5; x.b = 1 + rand() % 4;
    y.a = rand() % 3 ? x.a : 1 + rand() % 5; y.b = rand() % 3 ? x.b : 1 + rand() % 4;
    auto strides = [&](T& t) {
      const long inner = t.d + 8 * (rand() % 4), outer = rand() % 2 ? inner * (rand() % 2 ? t.b : t.a) : inner * t.b + 8 * (rand() % 6);
      if (rand() % 2) { t.sb = inner; t.sa = outer; } else { t.sa = inner; t.sb = outer; }
      if (t.sa < t.d) t.sa = t.d;
      if (t.sb < t.d) t.sb = t.d;
    };
    strides(x);
    if (rand() % 2) { y.sa = x.sa; y.sb = x.sb; } else strides(y);
    x.at = 1000000 + 16 * (rand() % 4); y.at = 1000000 + 16 * (rand() % 40);
    const std::set<long> p = bytes_of(x), q = bytes_of(y);
    bool meet = false;
    for (long v : p) meet = meet || q.count(v);
    auto range = [](const T& t) { return rows_of((const void*)t.at, t.a, t.sa, t.b, t.sb, t.d); };
    for (int two = 0; two < 2; ++two) {
      const bool got = two ? conflict({range(x), range(y)}, {}) : conflict({range(x)}, {range(y)});
      if (meet && !got) ++missed;
      if (!meet && got) ++refused;
      if (!meet && !got) ++taken;
    }
  }
  // K and V side by side per token, head by head, and head-major; output columns next to q, k, v in the rows of one buffer
  auto at = [](long x) { return (const void*)(4096 + 2 * x); };
  const long d = 64, H = 4, T_ = 10;
  const bool side = conflict({rows_of(at(0), T_, 2 * H * d, H, d, d), rows_of(at(H * d), T_, 2 * H * d, H, d, d)}, {});
  const bool inner = conflict({rows_of(at(0), T_, 2 * H * d, H, 2 * d, d), rows_of(at(d), T_, 2 * H * d, H, 2 * d, d)}, {});
  const bool major = conflict({rows_of(at(0), T_, 2 * d, H, 2 * T_ * d, d), rows_of(at(d), T_, 2 * d, H, 2 * T_ * d, d)}, {});
  const bool fused = conflict({rows_of(at(6 * d), T_, 10 * d, 4, d, d)},
                              {rows_of(at(0), T_, 10 * d, 4, d, d), rows_of(at(4 * d), T_, 10 * d, 1, d, d), rows_of(at(5 * d), T_, 10 * d, 1, d, d)});
  const bool over = conflict({rows_of(at(5 * d), T_, 10 * d, 4, d, d)}, {rows_of(at(5 * d), T_, 10 * d, 1, d, d)});
  std::printf("%ld %ld %ld %d %d %d %d %d\n", missed, refused, taken, side, inner, major, fused, over);
}
"""


def test_tensors_that_share_memory_byte_by_byte(tmp_path):
    """The check that stands before every call against the bytes themselves: what shares one is never taken, what alternates in one buffer is."""
    source, program = tmp_path / "harness.cpp", tmp_path / "harness"
    source.write_text(HARNESS)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-x", "c++", f"-I{CSRC}", str(source), "-o", str(program)])
    missed, refused, taken, side, inner, major, fused, over = map(int, subprocess.check_output([str(program)], text=True).split())
    assert missed == 0 and taken > refused
    assert (side, inner, major, fused, over) == (0, 0, 0, 0, 1)
