// Column sums of a matrix of fp32 partial results, in a fixed order: gradients of parameters, one row for each share of the
// tokens.  Sixteen teams of a workgroup take every sixteenth row of 64 columns, their sums are added in order: 512 rows of 8192
// columns 5 us (17 MB; with four teams 11, most of it waiting).
#include "mdh_internal.h"

namespace mdh {
namespace {

constexpr int kTeams = 16;
constexpr int64_t kColumns = (int64_t)1 << 27;  // of a launch: 2^31 lanes

struct SumArgs {
  const float* part;
  int64_t rows, n, first;  // columns, the launch's first one
  SumTarget to[3];
};

__global__ __launch_bounds__(64 * kTeams) void sum_rows_kernel(SumArgs s) {
  __shared__ float sums[kTeams][64];
  const int lane = threadIdx.x & 63, team = threadIdx.x >> 6;
  int64_t col = s.first + (int64_t)blockIdx.x * 64 + lane;
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  if (col < s.n) {
    const float* p = s.part + col;
    int64_t r = team;
    for (; r + 3 * kTeams < s.rows; r += 4 * kTeams)
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] += p[(r + u * kTeams) * s.n];
    for (; r < s.rows; r += kTeams) x[0] += p[r * s.n];
  }
  sums[team][lane] = (x[0] + x[1]) + (x[2] + x[3]);
  __syncthreads();
  if (team || col >= s.n) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < kTeams; ++k) v += sums[k][lane];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (col >= 0 && col < s.to[i].n && s.to[i].p) s.to[i].p[col] = v;
    col -= s.to[i].n;
  }
}

}  // namespace

mdh_status launch_sum_rows(const float* part, int64_t rows, int64_t n, const SumTarget (&to)[3], hipStream_t st) {
  if (!to[0].p && !to[1].p && !to[2].p) return MDH_OK;
  clear_stale_error();
  for (int64_t first = 0; first < n; first += kColumns) {
    const SumArgs s{part, rows, n, first, {to[0], to[1], to[2]}};
    sum_rows_kernel<<<(unsigned)cdiv(n - first < kColumns ? n - first : kColumns, 64), 64 * kTeams, 0, st>>>(s);
    const mdh_status r = launch_status();
    if (r != MDH_OK) return r;
  }
  return MDH_OK;
}

}  // namespace mdh
