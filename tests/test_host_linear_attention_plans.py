"""The linear-attention-block operators' choices of kernels, as the rules that they are compiled from say:
constant evaluation goes through the cases, in a syntax check of the host side. The sizes that the tests on
a device take to reach every kernel are here, with the kernel that each of them has to reach."""
import subprocess

import pytest

from paper_2008_03602_amd import _lib as L, build as B

# m, n, k, type of y, tiles, whether the reduction is split, rows and columns of launches of their own
TILES = [
    (20, 40, 200, "bf16", "32X16", 0, 0, 0), (20, 40, 200, "f32", "32X16", 0, 0, 0),
    (20, 24, 9000, "bf16", "32X16", 1, 0, 0), (20, 24, 9000, "f32", "32X16", 1, 0, 0),
    (40, 70, 200, "bf16", "32", 0, 0, 0), (40, 70, 200, "f32", "32", 0, 0, 0),
    (40, 70, 9000, "bf16", "32", 1, 0, 0), (40, 70, 9000, "f32", "32", 1, 0, 0),
    (1300, 1100, 96, "bf16", "64", 0, 0, 0), (1021, 1277, 200, "f32", "64", 0, 0, 0),
    (2000, 2010, 200, "bf16", "128X64", 0, 0, 0), (2000, 2010, 200, "f32", "128X64", 0, 0, 0),
    (2900, 2200, 168, "bf16", "128", 0, 0, 0), (2900, 2200, 168, "f32", "128", 0, 0, 0),
    (4096, 4099, 72, "f32", "128", 0, 0, 0),
    (4000, 3900, 168, "bf16", "256", 0, 0, 0), (3841, 4095, 72, "bf16", "256", 0, 0, 0),
    (4100, 4104, 72, "bf16", "256", 0, 4, 8),
]


def holds(tmp_path, unit):
    src = tmp_path / "unit.hip"
    src.write_text('#include "mx_linear_plan.h"\n' + unit)
    cmd = [B._hipcc()] + B.HIP_FLAGS + ["--offload-host-only", "-fsyntax-only", "-fconstexpr-steps=100000000", str(src)]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]


PLAN = r"""
constexpr ct::MxLinearPlan plan(int m, int n, int k, bool bf16) {
  ct_mx_linear_op op = {};
  op.m = m; op.n = n; op.k = k;
  op.x_format = op.w_format = CT_MX_E4M3;
  op.out_dtype = bf16 ? CT_DT_BF16 : CT_DT_F32;
  return ct::mx_linear_plan(op);
}
"""


def test_products_of_the_tests_reach_every_tile(tmp_path):
    checks = ["static_assert(%s(plan(%d, %d, %d, %d)), \"%s\");" % ("is<ct::MXL_%s, %d, %d, %d>" % (kind, split, tm, tn), m, n, k, out == "bf16",
                                                                  (m, n, k, out, kind))
              for m, n, k, out, kind, split, tm, tn in TILES]
    holds(tmp_path, PLAN + r"""
template <int KIND, bool SPLIT, int TAIL_M, int TAIL_N>
constexpr bool is(ct::MxLinearPlan p) {
  return p.kind == KIND && (p.split > 1) == SPLIT && (p.ws_floats > 0) == SPLIT && p.tail_m == TAIL_M && p.tail_n == TAIL_N;
}
""" + "\n".join(checks))
    assert {(t[3], t[4]) for t in TILES} >= {("f32", k) for k in ("32X16", "32", "64", "128X64", "128")}
    assert {t[4] for t in TILES if t[3] == "bf16"} == {"32X16", "32", "64", "128X64", "128", "256"}


def test_launches_apart_have_no_partial_sums_and_exact_sums_no_largest_tiles(tmp_path):
    holds(tmp_path, PLAN + r"""
constexpr bool sound() {
  const int sizes[] = {1, 16, 32, 33, 64, 65, 255, 256, 257, 300, 320, 512, 1000, 1024, 2048, 2100, 4096, 4100, 8192, 8200, 16385, 70000};
  for (int m : sizes)
    for (int n : sizes)
      for (int k : {0, 1, 128, 4096, 8192, 65536, 1 << 22})
        for (int bf16 = 0; bf16 < 2; ++bf16) {
          const ct::MxLinearPlan p = plan(m, n, k, bf16);
          if (p.kind < 0 || p.kind >= ct::MXL_KINDS || (!bf16 && p.kind == ct::MXL_256)) return false;
          if ((p.tail_m || p.tail_n) && (p.kind != ct::MXL_256 || p.split != 1 || p.ws_floats != 0)) return false;
          if (p.tail_m < 0 || p.tail_m > 64 || p.tail_n < 0 || p.tail_n > 64) return false;
          if ((p.tail_m && (m - p.tail_m) % 256) || (p.tail_n && (n - p.tail_n) % 256)) return false;
          // slices go over every step once, none of them empty
          const int64_t steps = ((int64_t)k + 127) / 128;
          if (p.split < 1 || (int64_t)p.split * p.per_split < steps) return false;
          if (p.split > 1 && (int64_t)(p.split - 1) * p.per_split >= steps) return false;
          if (p.ws_floats != (p.split > 1 ? (int64_t)p.split * m * ((n + 3) / 4 * 4) : 0)) return false;
        }
  return true;
}
static_assert(sound(), "");
""")


@pytest.mark.parametrize("m,n,k,out,kind,split,tm,tn", TILES)
def test_workspaces_are_as_the_plans_say(m, n, k, out, kind, split, tm, tn):
    op = L.make_mx_linear(m, n, k, L.MX_E4M3, L.MX_E2M1, L.DT_BF16 if out == "bf16" else L.DT_F32)
    assert (L.ct_mx_linear_workspace(op) > 0) == bool(split)
