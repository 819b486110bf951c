"""Which rows and columns the sequence-block kernels read, as the rules that they are compiled
from say: constant evaluation goes through the cases (and refuses a signed overflow), in a
syntax check of the host side."""
import subprocess

from paper_2008_03602_amd import build as B


def holds(tmp_path, unit):
    src = tmp_path / "unit.hip"
    src.write_text('#include "k_seq.h"\n' + unit)
    cmd = [B._hipcc()] + B.HIP_FLAGS + ["--offload-host-only", "-fsyntax-only", "-fconstexpr-steps=100000000", str(src)]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]


def test_lanes_without_a_state_read_columns_that_exist(tmp_path):
    # lanes of 4, 8 or 16 states, up to 16 of them a channel, over every row of whole quads
    holds(tmp_path, r"""
constexpr bool inside() {
  for (int states = 4; states <= 256; states += 4)
    for (int ns = 4; ns <= 16; ns *= 2)
      for (int part = 0; part < 16; ++part)
        for (int i = 0; i < ns; i += 4) {
          const int n = part * ns + i, col = ct::quad_column(n, states);
          if (col < 0 || col + 4 > states) return false;
          if (n < states && col != n) return false;
        }
  return true;
}
static_assert(inside(), "");
""")


def test_rows_asked_for_ahead_of_the_tokens_exist(tmp_path):
    # stages of TT tokens, U at a time, the next U asked for before these are walked: also after the last
    holds(tmp_path, r"""
constexpr bool inside(int tokens, int TT, int U) {
  for (int t = 0; t < tokens; t += TT) {
    const int rows = tokens - t < TT + U ? tokens - t : TT + U;
    for (int q = 0; q < TT + U; ++q) {
      const int row = ct::row_or_last(q, rows);
      if (row < 0 || t + row >= tokens) return false;
      if (t + q < tokens && row != q) return false;
    }
  }
  return true;
}
constexpr bool all_inside() {
  for (int tokens = 1; tokens <= 140; ++tokens)
    for (int TT : {4, 16, 32})
      for (int U : {4, 8})
        if (U <= TT && !inside(tokens, TT, U)) return false;
  return true;
}
static_assert(all_inside(), "");
""")


def test_copies_past_the_end_of_a_row_are_outside_by_any_range_check(tmp_path):
    # slices of 128 bytes of rows of `row` bytes, `have` rows `pitch` apart, also the slices past the
    # end; the check may look at the lane's offset alone or subtract the uniform one in 32 bits
    holds(tmp_path, r"""
constexpr bool sound(unsigned row, unsigned pitch, unsigned have, unsigned each) {
  const unsigned bytes = (have - 1) * pitch + row;
  for (unsigned k = 0; k < row + 3 * 128; k += 128)
    for (unsigned r = 0; r < have + 2; ++r)
      for (unsigned first = 0; first < 128; first += each) {
        const bool exists = k + first < row, mine = r < have;
        const unsigned lane = mine && exists ? r * pitch + first : ct::kOobGroup;
        const unsigned u = (unsigned)ct::uniform_part(k, bytes);
        const bool alone = lane < bytes, subtracted = lane < bytes - u;
        if (mine && exists) {
          if (!alone || !subtracted || lane + u != r * pitch + k + first || lane + u + each > bytes) return false;
        } else if (alone || subtracted) {
          return false;
        }
      }
  return true;
}
constexpr bool all_sound() {
  for (unsigned each : {4u, 16u})
    for (unsigned row = each; row <= 400; row += each)
      for (unsigned have : {1u, 2u, 5u})
        if (!sound(row, row, have, each) || !sound(row, row + 3 * each, have, each)) return false;
  return true;
}
static_assert(all_sound(), "");
""")


def test_tiles_end_within_their_sequence_up_to_the_most_rows(tmp_path):
    holds(tmp_path, r"""
constexpr int most = 0x7FFFFFFF - 4096;
constexpr bool ends(int begin, int end, int step) {
  for (int t = begin;; t = ct::tile_end(t, end, step)) {
    const int e = ct::tile_end(t, end, step);
    if (e < t || e > end || e - t > step || (e == t && t != end) || (e - t < step && e != end)) return false;
    if (e == end) return true;
  }
}
static_assert(ends(0, 0, 32) && ends(0, 1, 32) && ends(5, 37, 32) && ends(5, 38, 32) && ends(7, 1000, 8), "");
static_assert(ends(0, most, 262144) && ends(most - 1, most, 262144) && ends(most - 300000, most, 262144), "");
""")


def test_tile_numbers_that_no_rows_use_start_nowhere(tmp_path):
    # the last sequence is left with the numbers up to tokens / step, and with all of them where offsets do not ascend
    holds(tmp_path, r"""
constexpr int most = 0x7FFFFFFF - 4096;
constexpr bool starts(int tokens, int begin, int end, int step) {
  for (int k = 0; k <= tokens / step; k = k < 100 ? k + 1 : 2 * k) {
    const int t = ct::tile_start(begin, end, step, k);
    const bool used = (int64_t)begin + (int64_t)k * step < end || (k == 0 && begin == end);
    if (used ? t != begin + k * step : t != -1 && t != end) return false;
    if (begin == end && k > 0 && t != -1) return false;  // an empty sequence has one tile
  }
  const int last = ct::tile_start(begin, end, step, tokens / step);
  return last == -1 || (last >= begin && last <= end);
}
static_assert(starts(100, 0, 100, 8) && starts(100, 3, 50, 8) && starts(100, 60, 60, 8) && starts(96, 0, 96, 32), "");
static_assert(starts(most, 262143, most, 262144) && starts(most, 262143, most - 5, 262144), "");
static_assert(starts(most, most - 3, most, 8) && starts(most, most, most, 8) && starts(most, most - 9, most - 9, 262144), "");
""")


def test_tiles_are_counted_up_to_the_most_rows(tmp_path):
    holds(tmp_path, r"""
constexpr int most = 0x7FFFFFFF - 4096;
static_assert(ct::tiles_in(0, 32) == 0 && ct::tiles_in(1, 32) == 1 && ct::tiles_in(32, 32) == 1 && ct::tiles_in(33, 32) == 2, "");
static_assert(ct::tiles_in(most, 262144) == 8192 && ct::tiles_in(most, 8) == most / 8 + 1 && ct::tiles_in(most, most) == 1, "");
""")
