// Internal declarations of the operators on replica sets (prsgd_ops.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "prsgd_ops.h"

namespace prsgd {

// Sets the text of prsgd_last_error(NULL) of this thread and returns `code`.
int op_error(int code, const char* text);

constexpr int kMaxNormWidth = 16384;

struct NormArgs {
  const void* x; int64_t x_row;          // backward: dy
  const void* res; int64_t res_row;      // nullptr: none; backward: dsum
  const float* w; int64_t w_row;
  void* sum; int64_t sum_row;            // backward: s (read)
  void* y; int64_t y_row;                // rows of T, or bytes; backward: dx
  float* stat;                           // forward: rstd (may be nullptr) or scales; backward: rstd (read)
  float* dw; int64_t dw_row;             // backward: dw, or the workgroups' shares of it
  uint32_t rows, rows_per_worker;
  int width;
  float eps;
  int blocks;                            // backward: workgroups per worker
  bool streamed;                         // rows past the caches (filled in by the launcher)
};
hipError_t launch_rms_norm(NormArgs p, bool bf16, bool fp8, hipStream_t s);
// Workgroups per worker of the backward pass, and the floats of their shares of dw (0: a workgroup has its worker's rows to itself).
int norm_back_blocks(int workers, int64_t rows_per_worker, int width, bool bf16);
size_t norm_back_share_floats(int workers, int64_t rows_per_worker, int width, bool bf16);
hipError_t launch_rms_norm_backward(NormArgs p, float* shares, int workers, bool bf16, hipStream_t s);

// ---- orthogonalised updates ------------------------------------------------------------------

constexpr int kMaxOrthSide = 32768, kMaxOrthSteps = 64;
constexpr int kShortSide = 64;           // a side up to here goes through its Gram matrix in 64 bits
// Workgroups that sum a matrix's squares: enough to fill the device where a matrix is large.
constexpr int kMaxNormParts = 256;
constexpr int norm_parts(int rows, int cols) { return (int64_t)rows * cols < (1 << 20) ? 64 : kMaxNormParts; }
// Operands are halves of X, A and B times 2^13: entries reach 8, and what a second half holds of an entry of 2^-12 (X_0 of
// 4096 x 4096) is a normal number or loses less than 2^-36.
constexpr float kHalfScale = 8192.0f;
// Matrices whose norm is small beside eps give an X_0 that halves at this scale would hold in few bits or none (of norm 1e-5 at 1000 x 1000: ten
// bits).  X is stored 2^room times as large then, room being what |X_0| leaves below 1, and less by what the steps may have made of it:
// 2^max(0, room - grown[k]) in front of step k.  A and B need none of it, they are added to the coefficient a.
constexpr int kMostRoom = 100;           // an X_0 below 2^-100 loses bits again, as the result does in its own type from 2^-126 on

// What a call does with the matrices, whichever path computes.
struct OrthMatrices {
  const void* g; int64_t g_matrix, g_row;
  void* out; int64_t out_matrix, out_row;      // result, or (m != nullptr) the parameters that it updates
  float* m; int64_t m_matrix, m_row;           // momenta (nullptr: U = G)
  float mu, g_part, m_part;                    // M <- mu M + G, U = g_part G + m_part M
  float keep, step;                            // X <- keep X - step O
  int count, rows, cols;
  bool bf16;
  float eps, a, b, c;
  int steps;
};

// Storage of a matrix of halves [rows][ld]: rows of whole 128-byte lines.  Split (matrices of fp32): of every 16 columns the leading halves and then
// the remainders.
constexpr int half_ld(int cols, bool split) { return split ? (cols + 31) / 32 * 64 : (cols + 63) / 64 * 64; }
constexpr int half_rows(int rows) { return (rows + 63) / 64 * 64; }      // of X, which products contract over: padding rows hold zeros

// A product of every matrix, then an epilogue: acc = A B^T for the symmetric ones, A B for the others.
enum SquareEpilogue {
  SQ_GRAM = 0,    // out = acc (symmetric)
  SQ_POLY = 1,    // out = b lin + c acc (symmetric)
  SQ_NEXT = 2,    // out = a lin + acc
  SQ_LAST = 3,    // result = a lin + acc, into the caller's matrices
};
struct SquareArgs {
  const uint16_t* a; int64_t a_gs; int lda;
  const uint16_t* b; int64_t b_gs; int ldb;
  int M, N;
  const uint16_t* lin; const uint16_t* lin_lo; int64_t lin_gs; int ld_lin;     // lin_lo: remainders of unsplit X
  uint16_t* out; uint16_t* out_lo; int64_t out_gs; int ldo;
  uint16_t* out_t; int64_t t_gs; int ldt;      // where transposed tiles of a symmetric result go (out)
  const int* room;                             // per matrix
  float alpha, beta;                           // out = alpha lin + beta acc
  // Unsplit operands: B's diagonal, [M][2] per matrix: the half that the product takes and what it leaves out; both times diag_scale.
  float* diag; float diag_scale;
  int tiles_n, tiles;                          // per matrix; filled in by the launcher
  int count;
  bool transposed;                             // SQ_LAST: the caller's matrices hold the transpose
  uint8_t grown, grown_next;                   // of X in front of this step and behind it
  OrthMatrices user;
};
hipError_t launch_square(SquareArgs p, int epi, bool split, hipStream_t s);

hipError_t launch_orth_squares(const OrthMatrices& p, double* parts, hipStream_t s);
// X [half_rows(short side)][ld_x]; spare: where the next one goes, whose padding rows are cleared with it
struct OrthHalves { uint16_t* x; uint16_t* x_lo; uint16_t* spare; int64_t x_gs; int ld_x; int* room; };
hipError_t launch_orth_load(const OrthMatrices& p, const double* parts, const OrthHalves& h, hipStream_t s);
// Short sides: slices of the long side a matrix is cut into (1: one launch), and the doubles of a slice's Gram matrix.
int orth_short_slices(int count, int r, int longer);
size_t orth_short_doubles(int r);
hipError_t launch_orth_short(const OrthMatrices& p, double* grams, int slices, hipStream_t s);

}  // namespace prsgd
