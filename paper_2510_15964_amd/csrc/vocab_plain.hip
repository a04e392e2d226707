// Loss over a vocabulary with its gradients in single precision: the correctness configuration, sums in 64 bits, not tuned.  The
// logits of a piece of the tokens lie in the workspace as they are, and become G in place.
#include "../../include/lx.h"
#include "lx_dev.h"
#include "lx_launch.h"
#include "vocab.h"

namespace lx {

struct PlainPiece {
  int *n, *list, *target;      // tokens that have a target: how many, which, and theirs
  float* p;                    // [tokens][ldp]
  long long ldp;
  int first, count;
};

// One workgroup numbers the piece's tokens that have a target.
__global__ __launch_bounds__(1024) void plain_list(PlainVocabArgs a, PlainPiece q) {
  __shared__ int counts[16];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int before = 0;
  for (int t0 = 0; t0 < q.count; t0 += 1024) {
    const int t = t0 + (int)threadIdx.x, target = t < q.count ? a.targets[q.first + t] : -1;
    const unsigned long long held = __ballot((unsigned)target < (unsigned)a.V);
    if (lane == 0) counts[wave] = __popcll(held);
    __syncthreads();
    int at = before + __popcll(held & ((1ull << lane) - 1));
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += counts[w];
      before += counts[w];
    }
    if (held >> lane & 1) q.list[at] = q.first + t, q.target[at] = target;
    __syncthreads();
  }
  if (threadIdx.x == 0) *q.n = before;
}
// The other tokens' results.
__global__ __launch_bounds__(256) void plain_clear(PlainVocabArgs a, PlainPiece q) {
  const long long t = q.first + (int)blockIdx.x;
  if ((unsigned)a.targets[t] < (unsigned)a.V) return;
  if (threadIdx.x == 0) {
    a.loss[t] = 0.f;
    if (a.lse) a.lse[t] = 0.f;
  }
  if (a.dX)
    for (int c = threadIdx.x; c < a.d; c += 256) a.dX[t * a.dxs + c] = 0.f;
}

// out(m, n) = sum over k of left(m, k) right(n, k), a 64 x 64 tile to a workgroup, 4 x 4 results to a thread.  LK, RK: the operand lies
// with k contiguous.
template <bool LK, bool RK, class Left, class Right, class Out>
__device__ __forceinline__ void plain_product(int M, int N, int K, Left left, Right right, Out out) {
  __shared__ float l[16][65], r[16][65];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, x = threadIdx.x % 16, y = threadIdx.x / 16;
  if (m0 >= M) return;
  double sum[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = i * 256 + (int)threadIdx.x;
      const int lk = LK ? e % 16 : e / 64, lm = LK ? e / 16 : e % 64, rk = RK ? e % 16 : e / 64, rn = RK ? e / 16 : e % 64;
      l[lk][lm] = m0 + lm < M && k0 + lk < K ? left(m0 + lm, k0 + lk) : 0.f;
      r[rk][rn] = n0 + rn < N && k0 + rk < K ? right(n0 + rn, k0 + rk) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = fma((double)l[k][y + 16 * i], (double)r[k][x + 16 * j], sum[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (m0 + y + 16 * i < M && n0 + x + 16 * j < N) out(m0 + y + 16 * i, n0 + x + 16 * j, sum[i][j]);
}

__global__ __launch_bounds__(256) void plain_logits(PlainVocabArgs a, PlainPiece q) {
  plain_product<true, true>(*q.n, a.V, a.d, [&](int i, int c) { return a.X[q.list[i] * a.xs + c]; }, [&](int v, int c) { return a.W[(long long)v * a.d + c]; },
                            [&](int i, int v, double z) { q.p[i * q.ldp + v] = (float)z; });
}
// The loss of a token, and G in the place of its logits; the target's column apart, as in vocab.hip.
__global__ __launch_bounds__(256) void plain_rows(PlainVocabArgs a, PlainPiece q) {
  __shared__ double part[2][4];
  const int i = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (i >= *q.n) return;
  float* p = q.p + i * q.ldp;
  const int target = q.target[i];
  double top = -INFINITY, sum = 0;
  for (int v = threadIdx.x; v < a.V; v += 256) top = fmax(top, (double)p[v]);
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmax(top, __shfl_xor(top, o));
  if (lane == 0) part[0][wave] = top;
  __syncthreads();
  top = fmax(fmax(part[0][0], part[0][1]), fmax(part[0][2], part[0][3]));
  for (int v = threadIdx.x; v < a.V; v += 256)
    if (v != target) sum += exp((double)p[v] - top);
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) part[1][wave] = sum;
  __syncthreads();
  sum = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
  const double z = p[target], mine = exp(z - top), total = sum + mine;
  if (threadIdx.x == 0) {
    a.loss[q.list[i]] = (float)(mine > 0.5 * total ? log1p(sum / mine) : top - z + log(total));
    if (a.lse) a.lse[q.list[i]] = (float)(top + log(total));
  }
  if (!a.dX && !a.dW) return;
  __syncthreads();      // everybody has the target's logit
  const double w = a.weights ? a.weights[q.list[i]] : 1.f;
  for (int v = threadIdx.x; v < a.V; v += 256) p[v] = (float)(v == target ? -w * (sum / total) : w * (exp((double)p[v] - top) / total));
}
__global__ __launch_bounds__(256) void plain_dx(PlainVocabArgs a, PlainPiece q) {
  plain_product<true, false>(*q.n, a.d, a.V, [&](int i, int v) { return q.p[i * q.ldp + v]; }, [&](int c, int v) { return a.W[(long long)v * a.d + c]; },
                             [&](int i, int c, double x) { a.dX[q.list[i] * a.dxs + c] = (float)x; });
}
__global__ __launch_bounds__(256) void plain_dw(PlainVocabArgs a, PlainPiece q) {
  plain_product<false, false>(a.V, a.d, *q.n, [&](int v, int i) { return q.p[i * q.ldp + v]; }, [&](int c, int i) { return a.X[q.list[i] * a.xs + c]; },
                              [&](int v, int c, double x) {
                                float* to = a.dW + (long long)v * a.d + c;
                                *to = (float)(q.first == 0 ? x : x + (double)*to);
                              });
}

hipError_t launch_vocab_loss_plain(const PlainVocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st) {
  ProfScope prof(kKVocab, st);
  char* at = (char*)ws;
  PlainPiece q = {(int*)(at + room.head), (int*)(at + room.list), (int*)(at + room.target), (float*)(at + room.p), room.ldp, 0, 0};
  for (int t = 0; t < a.T; t += room.rows) {
    q.first = t;
    q.count = a.T - t < room.rows ? a.T - t : room.rows;
    const unsigned tiles = (q.count + 63) / 64, columns = (a.V + 63) / 64, width = (a.d + 63) / 64;
    hipError_t e = hipSuccess;
    auto launch = [&](auto kernel, dim3 grid, int threads) {
      if (e != hipSuccess) return;
      hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a, q);
      e = hipGetLastError();
    };
    launch(plain_list, dim3(1), 1024);
    launch(plain_clear, dim3(q.count), 256);
    launch(plain_logits, dim3(columns, tiles), 256);
    launch(plain_rows, dim3(q.count), 256);
    if (a.dX) launch(plain_dx, dim3(width, tiles), 256);
    if (a.dW) launch(plain_dw, dim3(width, columns), 256);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace lx
