// Internal interface of the gated linear recurrence (linear.hip) and the
// 4-bit gate products (q4.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

namespace alstm {

constexpr int kLinearSave = 8;     // timesteps between two saved states

// A gated linear recurrence, forward or back.  Layouts (row-major): p, dp
// [T][B][4H] (gate rows i, f, g, o), h, dh [T][B][H] of the call's type; c0,
// c_out, dc_out, dc0 [B][H], c_save [ceil(T/8)][B][H], bias, dbias [4H] fp32.
struct LinearArgs {
  const void* p;
  const float* bias;      // or null
  const int* lengths;     // [B] or null
  const float* c0;        // or null
  void* h;
  float* c_out;           // or null
  float* c_save;          // run: or null (written); backward: read
  const void* dh;
  const float* dc_out;    // or null
  void* dp;
  float* dc0;             // or null
  float* dbias;           // or null
  int T, B, H;
  int bf16;               // 1: p, h and their gradients hold bf16, else fp32
  int num_cu;
  // workspace (linear_workspace)
  float* dpart;           // [rows][4H]: sums of dp, one row per sequence (and stretch of time)
};

// Where the chunks of time of a column (64 pairs of units) hand over (linear.hip).
struct LinearScan {
  int cols, chunks, lanes;       // columns, chunks of time, pairs of units
  unsigned long long* maps;      // [chunks][lanes][2]: (A, B) of a unit
  unsigned* states;              // [groups][lanes][2]
  unsigned* tickets;             // [cols], 64 bytes apart
};

// Bytes of workspace of a run (backward 0), a backward pass (1) or one with the
// bias gradient (2).
size_t linear_workspace(int T, int B, int H, int num_cu, int backward);
// Whether a call of these sizes can be launched (4 B H below 2^30, T below 2^31 - 1024).
bool linear_fits(int T, int B, int H, int backward);
// Launches the recurrence, or its backward pass, with that workspace.
hipError_t launch_linear(const LinearArgs& a, void* ws, hipStream_t stream);
hipError_t launch_linear_backward(const LinearArgs& a, void* ws, hipStream_t stream);

// A matrix of 4-bit levels: the store's layout is described in q4.hip.
struct Q4Matrix {
  unsigned* q;        // [tiles][blocks][64][4]
  float* s;           // [tiles][padded][16]
  uint8_t* z;         // [tiles][padded][16]
  int R, D, G;
  int groups;         // of a row: ceil(D / G)
  int tiles;          // of 16 rows
  int blocks;         // of 128 columns
  int padded;         // groups of a padded row
};
// Sizes of a matrix; its bytes of device memory; its arrays' places there.
void q4_shape(Q4Matrix& m, int R, int D, int G);
size_t q4_bytes(const Q4Matrix& m);
void q4_place(Q4Matrix& m, uint8_t* store);
// Lays out q [R][ceil(D/2)], scale [R][groups], zero [R][groups] (null: 8) in m;
// *bad becomes 1 where a zero level is above 15.
hipError_t launch_q4_layout(const Q4Matrix& m, const uint8_t* q, const float* scale, const uint8_t* zero, int* bad,
                            hipStream_t stream);
// The opposite: the matrix in the formats of its layout's arguments.
hipError_t launch_q4_unpack(const Q4Matrix& m, uint8_t* q, float* scale, uint8_t* zero, hipStream_t stream);
// The kernel of a product and its shape: row tiles of a workgroup (of a wave in the
// tile kernel), rows of x (dot) or 16s of them, and waves, or halves of the columns
// (tile), that share the columns.
enum Q4Kernel { kQ4Dot, kQ4Rows, kQ4Tile };
struct Q4Form {
  Q4Kernel kernel;
  int tiles, x, split;
};
Q4Form q4_form(const Q4Matrix& m, int N, int bf16, int num_cu);
constexpr int kQ4MostRows = 1 << 20;   // of x in a launch (a grid's second dimension is short)
// y [N][R] = x [N][D] times the matrix, plus bias [R] (or null).
hipError_t launch_q4(const Q4Matrix& m, const void* x, int N, int bf16, const float* bias, void* y, int num_cu,
                     hipStream_t stream);

}  // namespace alstm
