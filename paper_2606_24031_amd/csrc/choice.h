// Which kernel a call takes, by its sizes and the device's compute units alone
// (host code without HIP, so that tests can ask it too).
#pragma once

#include <stdint.h>

namespace w4a8 {

// ------------------------------------------------------------------ q8q8_gemm
enum Q8Way { Q8_FEW_1x1, Q8_FEW_1x2, Q8_FEW_2x1, Q8_FEW_3x1, Q8_FEW_4x1,
             Q8_256x256, Q8_256x128, Q8_128x128, Q8_128x64, Q8_64x64, Q8_WAYS };

inline int q8_way(int64_t M, int64_t N, int cus) {
  // Up to 16 rows stream the weights; two tiles of channels a wave where there are
  // several rows and enough channels for all compute units eight times (16 rows over
  // 151936 x 2048 73 us against 89; one row 64 against 59).  Up to 64 rows do while
  // one workgroup a compute unit covers the channels (48 over 4096 x 2048 7.5 us, 8.4
  // on tiles; over 12288 x 2048 15, 9.2 on tiles).
  const int64_t n16 = (N + 15) / 16;
  if (M <= 16) return M > 1 && n16 >= 8 * cus ? Q8_FEW_1x2 : Q8_FEW_1x1;
  if (M <= 64 && n16 <= cus) return M <= 32 ? Q8_FEW_2x1 : M <= 48 ? Q8_FEW_3x1 : Q8_FEW_4x1;
  // One tile a compute unit takes `one`, each further round `more` (us at K = 2048): the
  // kind whose rounds end first.  It is the fastest of the five at K = 8192 too, at the
  // sizes below and 2000 x 4096, and at 512 the fastest or up to 9 % slower than it.
  // Measured at 2048:
  // 947 x 12288 37.5 on the largest tiles and 46, 45, 52, 62 on the others; 947 x
  // 8192 34, 29.5, 30.5, 38, 43; 947 x 4096 28, 23, 17, 19, 21; 947 x 2048 27, 22, 15,
  // 12, 12; 200 x 8192 27, 22, 15, 12, 11.5; 100 x 4096 26, 21, 14, 10.5, 8.4.
  struct Kind { int tn, tm; float one, more; };
  constexpr Kind kinds[] = {{256, 256, 30.f, 38.f}, {256, 128, 22.f, 25.f}, {128, 128, 14.f, 14.7f},
                            {128, 64, 10.5f, 8.7f}, {64, 64, 8.f, 5.1f}};
  int best = 0;
  float least = 0.0f;
  for (int i = 0; i < 5; i++) {
    const Kind &k = kinds[i];
    const int64_t tiles = ((N + k.tn - 1) / k.tn) * ((M + k.tm - 1) / k.tm);
    const float t = k.one + k.more * (float)((tiles - 1) / cus);
    if (i == 0 || t < least) { best = i; least = t; }
  }
  return Q8_256x256 + best;
}

// ------------------------------------------------------------------ ssm_scan
constexpr int SSM_CHUNK = 64;       // rows of a chunk
constexpr int SSM_STEP_T = 8;       // sequences of up to this many rows may go row by row,
constexpr int SSM_SPARE_T = 32;     // of up to this many in a plan with places to spare
constexpr int SSM_ORDER_B = 1024;   // up to this many are taken longest first by chunks

struct SsmWay {
  int rows;      // sequences of up to so many rows go row by row (0: none)
  bool single;   // ... one row at a time
  int chunked;   // so many sequences, the longest, go by chunks (0: none)
  int slice;     // columns of a workgroup by chunks
};

inline SsmWay ssm_way(int64_t B, int64_t T, int64_t NH, int64_t P, int N, int cus) {
  SsmWay w{};
  // Row by row, one launch, where no sequence can be long (8 rows), or hardly one:
  // exactly as many sequences as rows are taken to be a token each, and a chunk's
  // rows in a plan with places to spare are left to it too.  More rows in such a plan
  // may be one sequence's (947 of them, 64 heads of 64, in a plan of 1024: 1.11 ms row
  // by row, 0.11 by chunks, 0.04 in a plan of its own): there, up to 32 rows go row by
  // row, which takes what the chunks' launches do, and the others by chunks (1000
  // tokens in a plan of 1024: 802 us without those launches, 836 with them).
  // Batches that may hold many short sequences beside long ones: the short ones in
  // that launch too (16 of 4 rows: 22 us), the others chunk by chunk; few short ones
  // do not pay for a launch.
  w.single = T <= B;
  const bool all = T <= SSM_STEP_T || T == B || (w.single && T <= SSM_CHUNK);
  w.rows = all ? (int)T : w.single ? SSM_SPARE_T : T / SSM_CHUNK < B ? SSM_STEP_T : 0;
  if (all) return w;
  const int64_t most = T / (w.rows + 1);         // so many can have more rows
  w.chunked = (int)(B > SSM_ORDER_B || B < most ? B : most);
  // Slices of 32 columns read the records half as often as those of 16, which fill the
  // card with half the heads.  64 heads of 64, us: 2 sequences of 2000 rows 136 and
  // 136, 3 of them 219 and 201, 4 of them 235 and 257.
  w.slice = N == 64 || (N == 128 && w.chunked * NH * (P / 32) >= 2 * cus) ? 32 : 16;
  return w;
}

}  // namespace w4a8
