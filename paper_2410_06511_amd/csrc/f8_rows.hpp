// What the kernels that hold a row of a bf16 matrix in registers share (residual sums and norms), and the sums over their blocks.
#pragma once
#include <type_traits>

#include "f8_device.hpp"
#include "f8_host.hpp"

namespace f8 {

constexpr int64_t kRowMaxD = 16384;

// Kernels for THREADS == 64: a row per wave, four waves a block; above: a row per block of at most THREADS threads.
constexpr int kWaveRows = 4;
constexpr int block_threads(int THREADS) { return THREADS == kWave ? kWave * kWaveRows : THREADS; }

__device__ inline uint4 pack8(const float* f)
{
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ inline const uint4* row_of(const uint16_t* p, int64_t m, int64_t ld) { return reinterpret_cast<const uint4*>(p + m * ld); }
__device__ inline uint4* row_of(uint16_t* p, int64_t m, int64_t ld) { return reinterpret_cast<uint4*>(p + m * ld); }

// 1 / sqrt(v) rounded once: the fp64 instruction (some 2^-26 off) and one Newton step.  (Layer norm and the norm of a residual
// branch; the one after the residual sum has f8_rmsnorm's arithmetic and bits.)
__device__ inline float rsqrt_exact(double v)
{
    const double r = __builtin_amdgcn_rsq(v);
    return (float)(r > 0.0 && r < __builtin_inf() ? r + 0.5 * r * (1.0 - v * r * r) : r);
}

// Maximum over a block of any number of waves, for its first wave.
__device__ inline uint32_t waves_max(uint32_t v, uint32_t* red)
{
    v = wave_max_u32(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    return threadIdx.x < kWave ? wave_max_u32(threadIdx.x < blockDim.x / kWave ? red[threadIdx.x] : 0) : 0;
}

// ---- host ----

// f(upper bound of a block's threads, chunks a thread, threads): a row of dc chunks by as few waves as hold it with U chunks each
template <int T>
using Threads = std::integral_constant<int, T>;
template <class U, class F>
static void with_block(int64_t dc, U u, F&& f)
{
    const int threads = (int)((dc + u() * kWave - 1) / (u() * kWave)) * kWave;
    if (threads <= 256) f(Threads<256>{}, u, threads);
    else if (threads <= 512) f(Threads<512>{}, u, threads);
    else f(Threads<1024>{}, u, threads);
}
using One = std::integral_constant<int, 1>;
using Two = std::integral_constant<int, 2>;
template <class F>
static void with_row_shape(int64_t dc, F&& f)
{
    if (dc <= 64) f(Threads<64>{}, One{}, block_threads(64));
    else if (dc <= 128) f(Threads<64>{}, Two{}, block_threads(64));
    else with_block(dc, Two{}, f);
}
// Sums of the blocks' rows, in their order (f8_residual.hip): output row r < sets is that of part[r], the ones after it of part_gate.
constexpr int kSumCols = 32, kSumGroups = 16;
struct ColumnSums {
    const float* part[2];  // the gains' sums, one row a block
    float* out[2];
    int sets, strips;
    const float* part_gate;  // `parts` rows for each row of the gate
    float* dgate;
    int parts;
    int64_t D;
    const uint32_t* partial;  // nullable: the blocks' maxima
    int npartial;
    float* amax;
};
// rows: of outputs; nothing if there are no columns
void column_sums(const ColumnSums& p, unsigned rows, hipStream_t st);

}  // namespace f8
