// Microscaled 4-bit operands (OCP MX, E2M1 elements in blocks of 32 with an E8M0 scale): layout and launches that the linear's
// files share.
//   codes  [rows, pitch4(n)] bytes: element 2 i of a row in the low nibble of byte i; a row is padded with zeros to whole blocks
//   scales [groups of 512 elements][rows padded to 64][16] bytes: block b of the group's 16 at byte 4 (b % 4) + b / 4
// The scales' order is that of their use: the lane of a matrix instruction that holds elements 32 g .. 32 g + 31 of each 128
// finds those of four instructions in one word.  Bytes of no block hold 127, the scale 1.
#pragma once
#include "f8_host.hpp"

namespace f8 {

constexpr int kMxBlock = 32;    // elements with one scale
constexpr int kMxGroup = 512;   // elements of a scale group
constexpr int kMxRows = 64;     // rows of scales in a kilobyte
constexpr int64_t kMxMax = (int64_t)1 << 23;  // bound of M, K, N

__host__ __device__ inline int64_t mx4_pitch(int64_t n) { return (n + kMxBlock - 1) / kMxBlock * 16; }
__host__ __device__ inline int64_t mx4_rows(int64_t rows) { return (rows + kMxRows - 1) / kMxRows * kMxRows; }
inline size_t mx4_scale_bytes(int64_t rows, int64_t n) { return (size_t)((n + kMxGroup - 1) / kMxGroup) * (size_t)mx4_rows(rows) * 16; }

// Validated product D[M, N] = A[M, K] B[N, K]^T; a launch may take a part of it: the rows m0 .. M - 1, the columns n0 .. N - 1.
struct Mx4Args {
    int M, N, K;
    const uint8_t *A, *sa, *B, *sb;
    uint16_t* D;
    int64_t ldd;
    int m0 = 0, n0 = 0;                   // multiples of 256
    int64_t a_srows = mx4_rows(M), b_srows = mx4_rows(N);  // rows of the operands' scales
};
f8_status mx4_gemm(const Mx4Args& a, void* ws, size_t ws_bytes, hipStream_t st);
// The same of up to kMxTokens rows from their bf16 values [M, K] (a.A and a.sa unused), quantised inside: the same bits.
constexpr int kMxTokens = F8_MX4_TOKENS, kMxTokenK = F8_MX4_TOKEN_K;  // (their codes fit beside the ring in LDS)
f8_status mx4_gemm_tokens(const Mx4Args& a, const uint16_t* X, hipStream_t st);
size_t mx4_split_bytes(int64_t M, int64_t N, int64_t K);  // the most that a product takes of a workspace

}  // namespace f8
