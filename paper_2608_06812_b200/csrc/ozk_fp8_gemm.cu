// The block-scaled product C[m,n] = sum_k A(m,k) sa(m,k/128) B(n,k) sb(n,k/128) of E4M3 operands.
#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

struct Operand {
  const uint8_t* codes;
  int64_t ld;
  const void* scales;
  int kind, contract_rows;
  int lines;
  int64_t tiles;   // tiles per stored row of tiles (TILES kinds)
};

__device__ __forceinline__ float operand_scale(const Operand& o, int line, int b) {
  switch (o.kind) {
    case OZK_SCALE_LINES: return scale_value(static_cast<const uint8_t*>(o.scales)[((int64_t)(b / 4) * o.lines + line) * 4 + b % 4]);
    case OZK_SCALE_TILES: {
      const int64_t i = o.contract_rows ? (int64_t)b * o.tiles + line / kBlock : (int64_t)(line / kBlock) * o.tiles + b;
      return scale_value(static_cast<const uint8_t*>(o.scales)[i]);
    }
    case OZK_SCALE_LINES_F32: return static_cast<const float*>(o.scales)[(int64_t)line * o.tiles + b];
    default: return static_cast<const float*>(o.scales)[(int64_t)(line / kBlock) * o.tiles + b];
  }
}
__device__ __forceinline__ float operand_code(const Operand& o, int line, int k) {
  const uint8_t c = o.contract_rows ? o.codes[(int64_t)k * o.ld + line] : o.codes[(int64_t)line * o.ld + k];
  return unpack2(c).x;
}

// Plain form: one 32 x 32 tile of C per block, operands decoded into shared memory 32 values of k at a time.
template <class T>
__global__ void __launch_bounds__(256) product_kernel(Operand A, Operand B, int M, int N, int K, T* C, int64_t ldc, int accumulate) {
  __shared__ float a[32][33], b[32][33];
  const int m0 = blockIdx.y * 32, n0 = blockIdx.x * 32, tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  float sum[4] = {0.f, 0.f, 0.f, 0.f}, total[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < K; k0 += 32) {
    for (int i = ty; i < 32; i += 8) {
      // the thread index that runs fastest follows the contiguous axis of each operand
      const int la = A.contract_rows ? tx : i, ka = A.contract_rows ? i : tx;
      const int lb = B.contract_rows ? tx : i, kb = B.contract_rows ? i : tx;
      a[la][ka] = m0 + la < M && k0 + ka < K ? operand_code(A, m0 + la, k0 + ka) * operand_scale(A, m0 + la, (k0 + ka) / kBlock) : 0.f;
      b[lb][kb] = n0 + lb < N && k0 + kb < K ? operand_code(B, n0 + lb, k0 + kb) * operand_scale(B, n0 + lb, (k0 + kb) / kBlock) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 32; ++k)
      for (int j = 0; j < 4; ++j) sum[j] = fmaf(a[ty + 8 * j][k], b[tx][k], sum[j]);
    __syncthreads();
    if ((k0 + 32) % 8192 == 0 || k0 + 32 >= K)   // ranges of 8192, added in order
      for (int j = 0; j < 4; ++j) total[j] += sum[j], sum[j] = 0.f;
  }
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + ty + 8 * j, n = n0 + tx;
    if (m >= M || n >= N) continue;
    T* c = C + (int64_t)m * ldc + n;
    store_element(c, accumulate ? load_element(c) + total[j] : total[j]);
  }
}

bool check_operand(const ozk_fp8_operand* o, int64_t lines, int64_t k, Operand* out) {
  const int64_t cols = o->contract_rows ? lines : k;
  if (!o->codes || !o->scales || !aligned16(o->codes) || o->ld % 16 || o->ld < cols) return false;
  if (o->scale_kind < OZK_SCALE_LINES || o->scale_kind > OZK_SCALE_TILES_F32) return false;
  if (o->contract_rows != 0 && o->contract_rows != 1) return false;
  if (o->scale_kind != OZK_SCALE_TILES && (reinterpret_cast<uintptr_t>(o->scales) & 3)) return false;
  *out = Operand{o->codes, o->ld, o->scales, o->scale_kind, o->contract_rows, (int)lines, ceil_div(cols, kBlock)};
  return true;
}

constexpr size_t kGemmWorkspace = 24u << 20;

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

size_t ozk_fp8_gemm_workspace_bytes(void) { return kGemmWorkspace; }

ozk_status ozk_fp8_gemm(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, void* C, int c_type,
                        int64_t ldc, int accumulate, void* workspace, size_t workspace_size, void* stream) {
  if (M < 0 || N < 0 || K < 0 || !A || !B || ldc < N || (c_type != OZK_F32 && c_type != OZK_BF16) || (accumulate != 0 && accumulate != 1))
    return OZK_ERR_INVALID_ARG;
  if (M > INT32_MAX || N > INT32_MAX || K > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  if (accumulate && c_type != OZK_F32) return OZK_ERR_UNSUPPORTED;
  Operand a = {}, b = {};
  if (K > 0 && M > 0 && N > 0 && (!check_operand(A, M, K, &a) || !check_operand(B, N, K, &b))) return OZK_ERR_INVALID_ARG;
  const bool floats = a.kind >= OZK_SCALE_LINES_F32 || b.kind >= OZK_SCALE_LINES_F32;
  if (floats && (a.kind != OZK_SCALE_LINES_F32 || b.kind != OZK_SCALE_TILES_F32 || a.contract_rows || b.contract_rows))
    return OZK_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return OZK_OK;
  if (!C || (reinterpret_cast<uintptr_t>(C) & (c_type == OZK_F32 ? 3 : 1))) return OZK_ERR_INVALID_ARG;
  if (!workspace) workspace = workspace_ptr(), workspace_size = workspace_bytes();
  if (!workspace || workspace_size < kGemmWorkspace) return OZK_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)ceil_div(N, 32), (unsigned)ceil_div(M, 32));
  if (c_type == OZK_F32)
    product_kernel<<<grid, 256, 0, st>>>(a, b, (int)M, (int)N, (int)K, static_cast<float*>(C), ldc, accumulate);
  else
    product_kernel<<<grid, 256, 0, st>>>(a, b, (int)M, (int)N, (int)K, static_cast<__nv_bfloat16*>(C), ldc, 0);
  return cudaGetLastError() == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
}

}  // extern "C"
