// Which rows of h the LM heads read and which rows of z they write.
#pragma once
#include "scd_device.h"
#include "scd_kernels.h"

namespace scd {
namespace {

// Window rows are packed: row p = b * L + s of the B * L rows, blocks of 32 whatever the window length.
// row_dest: where window row p is stored, as a row of z [2, B, L] (ring slot (pos[b] + s) % L of half
// iter[b] & 1 when the decode state is given, else row p), or -1 if it is not live.  The kernels leave it
// in a table in LDS.  The two words of the state are fetched ahead of everything else and without a branch
// (from h where there is no state), so that nothing waits for them before they are used.
struct RowState {
  int p, b, p0, it;
};
__device__ __forceinline__ RowState row_state(const LmHeadArgs& a, int p) {
  const int q = min(p, a.B * a.L - 1);
  RowState r{p, q / a.L, 0, 0};
  const int32_t* const any = reinterpret_cast<const int32_t*>(a.h);
  r.p0 = (a.pos ? a.pos : any)[a.pos ? r.b : 0];
  r.it = (a.iter ? a.iter : any)[a.iter ? r.b : 0];
  return r;
}
__device__ __forceinline__ int row_dest(const LmHeadArgs& a, const RowState& r) {
  if (r.p >= a.B * a.L) return -1;
  if (!a.pos) return r.p;
  const int s = r.p - r.b * a.L, par = a.iter ? (r.it & 1) : 0;
  return s < a.N - r.p0 ? (par * a.B + r.b) * a.L + (r.p0 + s) % a.L : -1;
}
// First h row (of [B, C, L]) of the sequence that holds window row p.  A workgroup addresses its h rows from
// there: the whole of h may exceed the 4 GiB that a 32-bit offset reaches.
__device__ __forceinline__ int first_h_row(int p, int C, int L) { return p / L * C * L; }
// h row (of [B, C, L]) of row r < 32 of the block that starts at window row p0 (uniform; the last row where
// there is none: its results are not stored).  Windows of 32 or more positions end at most once in a block.
__device__ __forceinline__ int h_row(int p0, int r, int c, int C, int L, int rows) {
  int b = p0 / L, s = p0 - b * L + min(r, rows - 1 - p0);
  if (L >= 32) {
    const bool next = s >= L;
    b += next ? 1 : 0;
    s -= next ? L : 0;
  } else {
    const int w = s / L;
    b += w;
    s -= w * L;
  }
  return (b * C + c) * L + s;
}

template <int C>
__device__ __forceinline__ float processed_logit(const LmHeadArgs& a, float c, float u) {
  return scd::processed_logit<C>(a.lam, a.one_plus_lam, a.tau, c, u);
}

}  // namespace
}  // namespace scd
