// How the paged attention's work is split over workgroups: waves of a few-row
// workgroup, splits of the keys, workgroups of a launch. Host code alone.
#include <math.h>

#include <algorithm>

#include "zsa_internal.h"

namespace zsa {

bool paged_matrix(int dtype, int hd) { return dtype == 1 && hd >= 32; }

// Waves of a few-row workgroup: eight where the workgroups do not fill the CUs
// and every wave has more than two steps of 32 keys otherwise; one where short
// workgroups are many, and more of them run on a CU then (with four / one, us: 47
// sequences of up to 30 rows, 32 heads of 128, 14.6 / 8.9, of 250 27.9 / 25.9, 12 of
// 120 8.2 / 8.8; fp32, 47 of 30 36.6 / 16.4, 40 of 60, 32 of 128 on 8, 14.7 / 12.2,
// 60 of 250 27.3 / 30.9).
int paged_waves(bool matrix, int dtype, int hd, int tile, int max_len, int64_t workgroups) {
  const int cus = device_cu_count();
  if (tile == 16 && ((max_len <= 256 && workgroups * 2 >= cus * 5) || (!matrix && max_len <= 64 && workgroups > cus))) return 1;
  const bool can = matrix || (tile == 16 && hd * (dtype == 1 ? 2 : 4) <= 256);
  return can && max_len > 256 && workgroups <= cus ? 8 : 4;
}

// Keys that a few-row workgroup takes in one split (see paged_chunk).
static int paged_one(bool matrix, int hd, int64_t wgs, int64_t cus, int beside) {
  if (beside == 2 && matrix) return 512;
  if (beside == 0) {
    if (wgs * 5 >= cus * 7) return 2048;
    if (wgs <= cus && wgs * 16 >= cus * 11) return 4096;
    if (matrix && wgs <= cus) return hd == 128 && wgs * 4 < cus ? 1152 : 1536;
  }
  return matrix || 2 * wgs >= cus ? 1024 : 512;
}

// Splits of the keys; a second one needs the parts joined. `rows`: the packed
// ones of all key/value heads. `beside`: 1 with jobs
// of other sequences, 2 with a common prefix's.
//
// The few-row kernels: one for as many keys as a second would not pay its
// joining, 4 us and more (paged_one; us in one / two or three):
//  * 11/16 of the CUs or more, up to one each: 4096 keys (24 sequences of up to
//    3000 rows, 32 heads of 128 on 8, 48.8 / 55.6, of 8000 114 / 109; fp32, 25 of
//    4000, 111 / 107, 24 of 64 on 8 63.5 / 63.9);
//  * from 1.4 a CU: 2048 (64 of up to 1500, 32 of 128 on 8, 57.6 / 64, of 5000 181 /
//    185; fp32, 64 of 2000, 145 / 153);
//  * a few more than one a CU, which take twice as long as the rest: 1024 (40 of
//    up to 1500, 32 of 128 on 8, 46.5 / 43.3; fp32, 40 of 2000 117 / 107);
//  * fewer: 1536 (3 of up to 1500, 24 of 64 on 8, 11.3 / 12.3; 14 of 2000, 32 of 128
//    on 8, 26.5 / 24.2), in heads of 128 on less than a quarter of the CUs 1152 (6
//    of 1100 12.1 / 13.0, of 1500 15.0 / 13.5), in fp32 1024 or, under half of the
//    CUs, 512 (1 of 1000, 12 of 64, 19.8 / 15.2; 16 of up to 1024 21.0 / 21.6);
//  * beside a common prefix, where parts are joined in any case: in bf16 512 (20
//    of up to 900, 32 of 128, behind 900 46.2 / 43.7).
// Longer, of 512 keys at least, in fp32 of 256 where the CUs hold that many (2
// of up to 3089, 8 of 128 on 1, 15.4 / 21.0):
//  * few workgroups: one a CU, and not a few more than that, which would take
//    twice as long as the rest (4 sequences of 65536, 32 heads of 128 on 8, in
//    6, 8, 16, 31 splits 168, 156, 159, 164; 9 of up to 14000, 24 of 64 on 8, in 3, 4,
//    8 splits 49.6, 63.2, 48.4; 16 of up to 10000, 8 of 128 on 1, in 10, 16, 24
//    17.6, 17.6, 23.2);
//  * many: ragged sequences even out over a few splits each (64 of up to 4096, 32
//    of 128 on 8, in 1, 2, 4, 8 111, 109, 103, 105; 32 of up to 6000 in 1, 4, 6
//    89, 85, 92; 7 of 18000, 32 of 64, in 1, 4, 10 187, 191, 180), two beside other
//    jobs, whose rows would have as many parts.
//
// The many-row kernel, whose workgroups are long and few a CU: the number whose
// rounds over the CUs take least, with the parts' bytes. A workgroup takes 8 us
// and for 64 keys 1.1 us where few of its rows are there, 1.8 where all are, in
// heads below 128 1.4 to 2.6 where two are on a CU; parts are written and read at
// 2 TB/s, and a join that nothing else needs is 4 us. The sequences of a batch are
// taken as spread evenly from half of the longest on. Where the launch has `other`
// us of few-row work that fills the CUs between, the sum counts, not the rounds.
// (In 1, 2, 4 splits: 24 sequences of up to 2556 rows of which three bring 509, 32
// heads of 64, 62.3, 81.3, 93.5; 4 x 1024 over up to 8024, 32 of 128 on 8, 364, 420,
// 481; 16 questions on 4097 common rows, 32 of 64, in 2, 3, 4 77.3, 66.7, 69.4; 64 rows
// over 8192, 32 of 128 on 8, in 8, 11, 16 41.2, 36.2, 40.6; 12 x 20 over up to 3020, 24
// of 64 on 8, in 1, 2, 4, 6 64, 40, 27, 24. Over 80 such calls of 1 to 40 sequences it
// is 3% from the best number.)
int paged_chunk(bool many, bool matrix, int hd, int max_len, int64_t workgroups, int64_t rows, bool ragged, int beside, double other,
                int* splits) {
  const bool joined = beside > 0;
  const int64_t wgs = std::max<int64_t>(workgroups, 1), cus = std::max(device_cu_count(), 1);
  const int64_t small = static_cast<int64_t>(max_len + 255) / 256 * wgs;
  const int least = many || (!matrix && small <= cus) ? 256 : 512;
  const int64_t blocks = std::max(1, (max_len + least - 1) / least);
  int64_t want = 1;
  if (many) {
    const double part = static_cast<double>(rows) * hd * 8 / 2e6;
    const double full = std::min(1.0, static_cast<double>(rows) / (wgs * kPagedManyRows));
    double best = 0;
    for (int64_t n = 1; n <= std::min<int64_t>(blocks, 64); ++n) {
      const double chunk = static_cast<double>((blocks + n - 1) / n * least);
      const bool parts = n > 1 || joined;
      double each = 0;  // parts of a sequence
      for (int i = 0; i < 5; ++i) each += std::max(1.0, ceil((ragged ? 0.5 + 0.125 * i : 1) * max_len / chunk)) / 5;
      const double active = wgs * each;
      const int together = hd < 128 && active > cus ? 2 : 1;  // workgroups on a CU at a time
      const double rounds = active / (together * cus);
      const double len = ragged && (rounds > 1 || other > 0) ? 0.75 * max_len : max_len;
      const double one = std::min(chunk, len) * (together == 2 ? 1.4 + 1.2 * full : 1.1 + 0.7 * full) / 64 + 8;
      const double us = (other > 0 ? std::max(one, rounds * one + other) : ceil(rounds) * one) + (parts ? n * part : 0) +
                        (parts && !joined ? 4 : 0);
      if (n == 1 || us < best) {
        best = us;
        want = n;
      }
    }
  } else if (max_len > paged_one(matrix, hd, wgs, cus, beside)) {
    if (wgs * 16 < cus * 11) {
      want = (cus * 15 / 16 + wgs - 1) / wgs;
      if (wgs * want > cus && wgs * (want - 1) * 32 >= cus * 25) --want;
    } else {
      want = joined || !matrix ? 2 : std::max(4, std::min(max_len / 1800, 10));
    }
    want = std::min(want, blocks);
  }
  const int per = static_cast<int>((blocks + want - 1) / want);
  *splits = static_cast<int>((blocks + per - 1) / per);
  return per * least;
}

int64_t paged_blocks(const PagedAttention& a, bool many) {
  const int64_t pairs = static_cast<int64_t>(a.splits) * (a.H / a.G) * a.B;
  return (many ? (pairs + 7) / 8 * 8 : pairs) * a.tiles;
}

}  // namespace zsa
