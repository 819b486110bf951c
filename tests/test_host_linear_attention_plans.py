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


def holds(tmp_path, unit, header="mx_linear_plan.h"):
    src = tmp_path / "unit.hip"
    src.write_text('#include "%s"\n' % header + unit)
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


def test_pieces_of_bad_offsets_have_places_of_their_own(tmp_path):
    """A sequence's pieces are numbered from first_tile on. Whatever the offsets hold, the places of its pieces,
    the last one's too, are below the total that workspaces are sized by; where the offsets ascend no two
    sequences have one in common, and every row lies in one piece."""
    holds(tmp_path, r"""
constexpr unsigned next(unsigned& seed) { return seed = seed * 1664525u + 1013904223u, seed >> 8; }
constexpr bool inside() {
  unsigned seed = 3;
  for (int round = 0; round < 3000; ++round) {
    const int count = 1 + next(seed) % 7, step = 64 * (1 + next(seed) % 4), tokens = next(seed) % 3000;
    const bool ascend = next(seed) % 2;
    int offsets[8] = {}, last = 0;
    for (int i = 0; i <= count; ++i) {
      const unsigned kind = next(seed) % 6;
      if (ascend) offsets[i] = last = last + (kind ? (int)(next(seed) % (tokens - last + 1)) / 2 : 0);
      else offsets[i] = kind == 0 ? -2147483647 - 1 : kind == 1 ? 2147483647 : (int)(next(seed) % (tokens + 200)) - 100;
    }
    const ct::SeqView view = {offsets, nullptr, tokens, count, count, 0};
    const int64_t total = ct::seq_tiles(view, step).total;
    int64_t behind = 0;  // the first number that no sequence so far has
    for (int s = 0; s < count; ++s) {
      const int begin = ct::seq_row(offsets[s], 0, tokens), end = ct::seq_row(offsets[s + 1], begin, tokens);
      if (begin < 0 || begin > end || end > tokens) return false;
      const int first = ct::first_tile(begin, step, s), tiles = ct::tiles_in(end - begin, step), owned = tiles ? tiles : 1;
      if (first < 0 || first + owned > total || (ascend && first < behind)) return false;
      behind = first + owned;
      int row = begin;
      for (int k = 0; k < tiles; ++k) {
        const int at = ct::tile_start(begin, end, step, k);
        if (at != row || at >= end) return false;
        row = ct::tile_end(at, end, step);
      }
      if (row != end || ct::tile_start(begin, end, step, tiles + 1) >= 0) return false;
    }
  }
  return true;
}
static_assert(inside(), "");
constexpr bool equal_lengths() {
  for (int len : {0, 1, 63, 64, 65, 1000, 1 << 29})
    for (int step : {64, 256})
      for (int count : {0, 1, 3}) {
        const ct::SeqView view = {nullptr, nullptr, len * count, count, count, len};
        const ct::SeqTiles t = ct::seq_tiles(view, step);
        if (t.per < 1 || t.total != (int64_t)t.per * count || (int64_t)t.per * step < len) return false;
      }
  return true;
}
static_assert(equal_lengths(), "");
""", "k_seq.h")


def test_workspaces_of_attention_hold_every_piece():
    """The library's own answer: a state and a decay for each head and piece, for as many pieces as it takes."""
    for tokens, count, heads, key, value in ((65536, 1, 2, 128, 128), (600, 1, 2, 250, 130), (4096, 3, 4, 64, 64), (70000, 1000, 1, 8, 8)):
        op = L.make_decay_attention(heads, heads, key, value, L.DT_BF16)
        need = L.ct_decay_attention_workspace(op, L.make_sequences(tokens, count, count, tokens, 0x1000))
        dk = 64 if key <= 64 else 128 if key <= 128 else 256
        columns = -(-value // 64) * 64 if value <= 64 or dk == 256 else -(-value // 128) * 128
        each = 4 * heads * (dk * columns + 1)
        assert need > 0 and need % each == 0
        pieces = need // each - count  # tokens / piece
        assert 1 <= pieces <= tokens // 64


def test_attention_refuses_a_workspace_that_is_too_small():
    ok = 0x1000
    op, seqs = L.make_decay_attention(2, 2, 128, 128, L.DT_BF16), L.make_sequences(65536, 1, 1)
    need = L.ct_decay_attention_workspace(op, seqs)
    assert need > 0
    for ws, have, what in ((None, 0, "workspace"), (ok, need - 1, "workspace"), (ok + 8, need, "16-byte")):
        with pytest.raises(L.CtError) as e:
            L.ct_decay_attention_run(op, seqs, ok, ok, ok, ok, ok, ok, ok, ok, ok, ws=ws, ws_bytes=have)
        assert e.value.code == L.CT_E_ARG and what in str(e.value)
