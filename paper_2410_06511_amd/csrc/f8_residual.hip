// The residual sum of a transformer block's branch with the norms before and after it, forward and backward:
//   u = y r1 g_post (or y),  r1 = 1 / sqrt(mean y^2 + eps);   h = bf16(a x + b gate u);   n = h r2 g_pre,  r2 of the rounded h;
//   t = dh + r2 g_pre dn - h r2^3 mean(h g_pre dn),  dx = a t,  v = b gate t,  dy = r1 g_post v - y r1^3 mean(y g_post v) (or v),
//   dgate = sum over its rows of b t u,  dg_post = sum v y r1,  dg_pre = sum dn h r2.
// Bound by memory: 8 bytes an element forward (x, y -> h, n), 12 backward (h, y, dh, dn -> dx, dy); as separate calls the sum,
// the gate and each norm read and write their tensors again.  16384 x 8192 with both norms and gates: forward 190 us (5.6 TB/s),
// backward 318 and 7 for its sums (5.0); 8192 x 4096 with the norm after the sum only: 44 (6.1), 58 and 5 (5.3).
// A row is held in registers by TPR threads, U chunks of 16 bytes each, so that every tensor is read once although a norm needs
// its row twice.  Sums over a row are taken in f8_rmsnorm's order (chunks 64 apart one after the other, then lanes by halves), so
// that the plain residual and norm have the bits of f8_add followed by f8_rmsnorm.  Sums over rows have a fixed order too.
#include "f8_device.hpp"
#include "f8_host.hpp"
#include "f8_rows.hpp"

namespace f8 {

constexpr int kResBlocks = 2048;     // of the forward: one partial maximum each
// Blocks of the backward, each of which leaves a partial row of every gain's sums (4096 x 4096 with 256 / 512 blocks 58 / 53 us,
// 768 71); half as many above 4096 elements a row, where a block's waves fill a compute unit (16384 x 8192 371 -> 341 us, 300 x 8192
// 26 -> 22).
constexpr int kResBwdBlocks = 512;
// Elements from which the backward loads past the caches (16384 x 8192 348 -> 326 us, 12288 x 4096 115 -> 92, 8192 x 5120 126 -> 118;
// at the limit, 8192 x 4096, 65 -> 64; 4096 x 4096 52 -> 53, 2001 x 2816 26 -> 27).
constexpr int64_t kResOnce = (int64_t)1 << 25;
static_assert((size_t)kResBlocks * sizeof(uint32_t) <= kMinWorkspaceBytes, "one partial per block fits the minimum workspace");

struct ResidualArgs {
    const uint16_t *x, *y;
    int64_t ldx, ldy;
    const uint4 *g_post, *gate, *g_pre;
    int64_t M, per_gate;  // rows that share a row of the gate
    int dc;               // 16-byte chunks of a row
    float a, b, eps, inv_d;
    double inv_d64;
    uint16_t *h, *n;
    int64_t ldh, ldn;
    float *rstd_post, *rstd_pre;
    uint32_t* partial;
};

// Sum over a wave in f8_rmsnorm's order; a row waits for it up to twice.
__device__ inline float wave_sum(float v)
{
    return wave_all(v, [](float a, float b) { return a + b; });
}

// Sum over a row of the chunks' terms; thread t of the row's TPR has chunks t, t + TPR, ...  Two buffers in turn and one barrier:
// a buffer is written again only after the barrier of the sum in between.
template <int THREADS, int U>
struct RowSum {
    static constexpr int kPieces = THREADS > kWave ? THREADS / kWave * U : 1;
    float (*terms)[kPieces][kWave];
    int buf = 0;
    __device__ float operator()(const float* term)
    {
        const int lane = threadIdx.x & (kWave - 1);
        float s = 0.0f;
        if constexpr (THREADS == kWave) {
#pragma unroll
            for (int u = 0; u < U; ++u) s += term[u];
        } else {
            const int wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
#pragma unroll
            for (int u = 0; u < U; ++u) terms[buf][wave + waves * u][lane] = term[u];
            __syncthreads();
#pragma unroll 8
            for (int i = 0; i < waves * U; ++i) s += terms[buf][i][lane];
            buf ^= 1;
        }
        return wave_sum(s);
    }
};

template <int THREADS, int U, bool POST, bool PRE>
__global__ __launch_bounds__(block_threads(THREADS)) void residual_norm_kernel(const ResidualArgs p)
{
    constexpr int kRows = THREADS == kWave ? kWaveRows : 1;
    __shared__ float terms[2][RowSum<THREADS, U>::kPieces][kWave];
    __shared__ uint32_t red[block_threads(THREADS) / kWave];
    RowSum<THREADS, U> sum{terms};
    const int TPR = THREADS == kWave ? kWave : (int)blockDim.x, t = THREADS == kWave ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    uint32_t mag = 0;
    for (int64_t m0 = (int64_t)blockIdx.x * kRows; m0 < p.M; m0 += (int64_t)gridDim.x * kRows) {
        const int64_t m = m0 + (THREADS == kWave ? (int)threadIdx.x / kWave : 0);
        const bool live = m < p.M;
        uint4 x[U], y[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            in[u] = live && c < p.dc;
            x[u] = y[u] = make_uint4(0, 0, 0, 0);
            if (in[u]) x[u] = row_of(p.x, m, p.ldx)[c], y[u] = row_of(p.y, m, p.ldy)[c];
        }
        float r1 = 1.0f, term[U];
        if constexpr (POST) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
                unpack8(y[u], f);
                term[u] = ((f[0] * f[0] + f[1] * f[1]) + (f[2] * f[2] + f[3] * f[3])) + ((f[4] * f[4] + f[5] * f[5]) + (f[6] * f[6] + f[7] * f[7]));
            }
            r1 = rsqrt_exact((double)sum(term) * p.inv_d64 + (double)p.eps);
            if (p.rstd_post && t == 0 && live) p.rstd_post[m] = r1;
        }
        const uint4* gate = p.gate && live ? p.gate + (int64_t)((uint32_t)m / (uint32_t)p.per_gate) * p.dc : nullptr;
        uint4 h[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            float fx[8], fy[8], g[8];
            unpack8(x[u], fx), unpack8(y[u], fy);
            if (POST && in[u]) {
                unpack8(p.g_post[c], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) fy[j] = (fy[j] * r1) * g[j];
            }
            if (gate && in[u]) {
                unpack8(gate[c], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) fy[j] = g[j] * fy[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) fx[j] = p.a * fx[j] + p.b * fy[j];
            h[u] = pack8(fx);
            if (in[u]) row_of(p.h, m, p.ldh)[c] = h[u];
            if (!in[u]) h[u] = make_uint4(0, 0, 0, 0);
        }
        if constexpr (PRE) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
                unpack8(h[u], f);
                term[u] = ((f[0] * f[0] + f[1] * f[1]) + (f[2] * f[2] + f[3] * f[3])) + ((f[4] * f[4] + f[5] * f[5]) + (f[6] * f[6] + f[7] * f[7]));
            }
            const float r2 = 1.0f / sqrtf(sum(term) * p.inv_d + p.eps);
            if (p.rstd_pre && t == 0 && live) p.rstd_pre[m] = r2;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!in[u]) continue;
                const int c = t + TPR * u;
                float f[8], g[8];
                unpack8(h[u], f), unpack8(p.g_pre[c], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = (f[j] * r2) * g[j];
                const uint4 o = pack8(f);
                row_of(p.n, m, p.ldn)[c] = o;
                mag = absmax_acc(mag, o);
            }
        }
    }
    if (PRE && p.partial) {
        const uint32_t mx = waves_max(pk_collapse(mag), red);
        if (threadIdx.x == 0) p.partial[blockIdx.x] = mx;
    }
}

// ---- backward ----------------------------------------------------------------------------------

struct ResidualGradArgs {
    const uint16_t *h, *y, *dh, *dn;  // h with PRE, y with POST or a gate; dh nullable with PRE
    int64_t ldh, ldy, lddh, lddn;
    const uint4 *g_post, *gate, *g_pre;
    const float *rstd_post, *rstd_pre;
    int64_t M, per_gate, units;
    int parts, dc;
    float a, b, inv_d;
    uint16_t *dx, *dy;  // nullable
    int64_t lddx, lddy;
    float *part_pre, *part_post, *part_gate;  // [block][D], [unit][D] (the gate's own gradient where a unit is a whole group)
    uint32_t* partial;
};

// A block takes units: the rows part, part + parts, ... of one group of rows that share a gate's row, and leaves one row of
// sums a gain.
template <int THREADS, int U, bool POST, bool GATE, bool PRE, bool ONCE>
__global__ __launch_bounds__(block_threads(THREADS)) void residual_norm_bwd_kernel(const ResidualGradArgs p)
{
    constexpr int kRows = THREADS == kWave ? kWaveRows : 1;
    __shared__ float terms[2][RowSum<THREADS, U>::kPieces][kWave];
    __shared__ float share[kRows][kRows > 1 ? kWave * U * 8 : 1];
    __shared__ uint32_t red[block_threads(THREADS) / kWave];
    RowSum<THREADS, U> sum{terms};
    const int TPR = THREADS == kWave ? kWave : (int)blockDim.x;
    const int t = THREADS == kWave ? (int)threadIdx.x % kWave : (int)threadIdx.x, sub = THREADS == kWave ? (int)threadIdx.x / kWave : 0;
    uint32_t mag = 0;
    float acc_pre[U][8] = {}, acc_post[U][8] = {};
    struct Row {
        uint4 h[U], y[U], dh[U], dn[U];
        float r1, r2;
    };
    // out[D] = sum over the block's row slots of acc, in their order
    auto leave = [&](float (*acc)[8], float* out) {
        if constexpr (kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) share[sub][(u * 8 + j) * kWave + t] = acc[u][j];
            __syncthreads();
            if (sub) return;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float s = share[0][(u * 8 + j) * kWave + t];
                    for (int k = 1; k < kRows; ++k) s += share[k][(u * 8 + j) * kWave + t];
                    acc[u][j] = s;
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            if (c >= p.dc) continue;
            float* o = out + (int64_t)c * 8;  // (a caller's dgate lies on any word)
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = acc[u][j];
        }
    };
    for (int64_t unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const int64_t group = unit / p.parts, part = unit - group * p.parts;
        const int64_t first = group * p.per_gate, rows = (p.per_gate - part + p.parts - 1) / p.parts;  // of this unit
        const uint4* gate = GATE ? p.gate + group * p.dc : nullptr;
        float acc_gate[U][8] = {};
        for (int64_t k0 = 0; k0 < rows; k0 += kRows) {
            const int64_t k = k0 + sub, m = first + part + k * p.parts;
            const bool live = k < rows;
            Row row;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = t + TPR * u;
                row.h[u] = row.y[u] = row.dh[u] = row.dn[u] = make_uint4(0, 0, 0, 0);
                if (!live || c >= p.dc) continue;
                const auto load = [&](const uint16_t* t, int64_t ld) { return ONCE ? load_once(row_of(t, m, ld) + c) : row_of(t, m, ld)[c]; };
                if (PRE) row.h[u] = load(p.h, p.ldh), row.dn[u] = load(p.dn, p.lddn);
                if (POST || GATE) row.y[u] = load(p.y, p.ldy);
                if (!PRE || p.dh) row.dh[u] = load(p.dh, p.lddh);
            }
            row.r1 = POST && live ? p.rstd_post[m] : 0.0f;
            row.r2 = PRE && live ? p.rstd_pre[m] : 0.0f;
            float term[U], dt[U][8];
            if constexpr (PRE) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = t + TPR * u;
                    float fh[8], fd[8], g[8];
                    unpack8(row.h[u], fh), unpack8(row.dn[u], fd), unpack8(p.g_pre[c < p.dc ? c : 0], g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        acc_pre[u][j] += fd[j] * (fh[j] * row.r2);
                        dt[u][j] = g[j] * fd[j];
                        g[j] = fh[j] * dt[u][j];
                    }
                    term[u] = ((g[0] + g[1]) + (g[2] + g[3])) + ((g[4] + g[5]) + (g[6] + g[7]));
                }
                const float k2 = row.r2 * (row.r2 * (row.r2 * (sum(term) * p.inv_d)));  // (r^3 alone could underflow)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float fh[8], fd[8];
                    unpack8(row.h[u], fh), unpack8(row.dh[u], fd);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dt[u][j] = fd[j] + (row.r2 * dt[u][j] - fh[j] * k2);
                }
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) unpack8(row.dh[u], dt[u]);
            }
            if (p.dx) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = t + TPR * u;
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = p.a * dt[u][j];
                    if (live && c < p.dc) store_stream(row_of(p.dx, m, p.lddx) + c, pack8(o));
                }
            }
            // from here on dt is the gradient of u
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = t + TPR * u, cc = c < p.dc ? c : 0;
                float fy[8], g[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) dt[u][j] *= p.b;
                if constexpr (POST || GATE) unpack8(row.y[u], fy);
                if constexpr (GATE) {
                    float gp[8], gg[8];
                    unpack8(gate[cc], gg);
                    if constexpr (POST) unpack8(p.g_post[cc], gp);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        acc_gate[u][j] += dt[u][j] * (POST ? (fy[j] * row.r1) * gp[j] : fy[j]);
                        dt[u][j] *= gg[j];
                    }
                }
                if constexpr (POST) {
                    unpack8(p.g_post[cc], g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        acc_post[u][j] += dt[u][j] * (fy[j] * row.r1);
                        dt[u][j] *= g[j];
                        g[j] = fy[j] * dt[u][j];
                    }
                    term[u] = ((g[0] + g[1]) + (g[2] + g[3])) + ((g[4] + g[5]) + (g[6] + g[7]));
                }
            }
            if constexpr (POST) {
                const float k1 = row.r1 * (row.r1 * (row.r1 * (sum(term) * p.inv_d)));
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float fy[8];
                    unpack8(row.y[u], fy);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dt[u][j] = row.r1 * dt[u][j] - fy[j] * k1;
                }
            }
            if (p.dy) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = t + TPR * u;
                    const uint4 o = pack8(dt[u]);
                    if (live && c < p.dc) {
                        store_stream(row_of(p.dy, m, p.lddy) + c, o);
                        mag = absmax_acc(mag, o);
                    }
                }
            }
        }
        if (GATE && p.part_gate) leave(acc_gate, p.part_gate + unit * p.dc * 8);
    }
    if (PRE && p.part_pre) leave(acc_pre, p.part_pre + (int64_t)blockIdx.x * p.dc * 8);
    if (POST && p.part_post) leave(acc_post, p.part_post + (int64_t)blockIdx.x * p.dc * 8);
    if (p.partial) {
        const uint32_t mx = waves_max(pk_collapse(mag), red);
        if (threadIdx.x == 0) p.partial[blockIdx.x] = mx;
    }
}

// The sums of the blocks' rows, in their order: blockIdx.y is a set of `strips` rows of partial sums and its output row.
__global__ __launch_bounds__(kSumCols* kSumGroups) void column_sums_kernel(const ColumnSums p)
{
    __shared__ float sum[kSumGroups][kSumCols];
    __shared__ uint32_t red[kSumGroups * kSumCols / kWave];
    const int cl = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols;
    const int64_t c = (int64_t)blockIdx.x * kSumCols + cl;
    const int set = (int)blockIdx.y, n = set < p.sets ? p.strips : p.parts;
    const float* src = set < p.sets ? p.part[set] : p.part_gate + (int64_t)(set - p.sets) * p.parts * p.D;
    float* out = set < p.sets ? p.out[set] : p.dgate + (int64_t)(set - p.sets) * p.D;
    float s = 0.0f;
    if (c < p.D) {
        int i = grp;
        const auto batch = [&](auto ahead) {  // that many rows' loads at once
            constexpr int AHEAD = decltype(ahead)::value;
            float v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int at = i + kSumGroups * k;
                v[k] = at < n ? src[(int64_t)at * p.D + c] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) s += v[k];
            i += kSumGroups * AHEAD;
        };
        while (i + kSumGroups * 31 < n) batch(std::integral_constant<int, 32>{});
        while (i < n) batch(std::integral_constant<int, 8>{});
    }
    sum[grp][cl] = s;
    __syncthreads();
    if (grp == 0 && c < p.D) {
        float v = sum[0][cl];
#pragma unroll
        for (int k = 1; k < kSumGroups; ++k) v += sum[k][cl];
        out[c] = v;
    }
    if (p.amax && blockIdx.x == 0 && set == 0) {
        uint32_t m = 0;
        for (int i = threadIdx.x; i < p.npartial; i += kSumGroups * kSumCols) m = p.partial[i] > m ? p.partial[i] : m;
        m = block_max_u32<kSumGroups * kSumCols / kWave>(m, red);
        if (threadIdx.x == 0) p.amax[0] = mag_to_float(m);
    }
}

void column_sums(const ColumnSums& p, unsigned rows, hipStream_t st)
{
    column_sums_kernel<<<dim3((unsigned)((p.D + kSumCols - 1) / kSumCols), rows), kSumCols * kSumGroups, 0, st>>>(p);
}

// ---- host ----------------------------------------------------------------------------------------

// The backward holds four rows and up to three rows of sums.  One chunk a thread leaves registers for enough waves up to 8192
// elements (16384 x 8192 394 -> 371 us, 8192 x 2048 59 -> 50), but a row of 520 to 1024 elements is better a wave's own, without
// barriers (8192 x 1024 45 -> 30); with a norm of the branch the two are within 6 % between 2816 and 4096 (2001 x 2816 26.9 -> 25.8,
// 8192 x 2816 66 -> 70).  Waves hide the loads better than loads ahead of the row, which take their registers (4096 x 4096
// 74 -> 53).
template <class F>
static void with_bwd_shape(int64_t dc, F&& f)
{
    if (dc <= 64) f(Threads<64>{}, One{}, block_threads(64));
    else if (dc <= 128) f(Threads<64>{}, Two{}, block_threads(64));
    else if (dc <= 1024) with_block(dc, One{}, f);
    else f(Threads<1024>{}, Two{}, (int)((dc + 2 * kWave - 1) / (2 * kWave)) * kWave);
}

// How the backward divides its rows: `parts` blocks share a group of rows with one gate row while there are fewer groups than
// blocks, else a block takes whole groups.
struct ResidualPlan {
    int64_t per_gate, units;
    int parts, blocks;
};
static ResidualPlan plan_bwd(int64_t M, int64_t D, int64_t gate_rows)
{
    const int64_t groups = gate_rows > 0 ? gate_rows : 1, per_gate = M / groups, slots = D / 8 <= 128 ? kWaveRows : 1;  // rows that a block takes at once
    const int blocks = D / 8 > 512 ? kResBwdBlocks / 2 : kResBwdBlocks;
    int64_t parts = blocks / groups, most = (per_gate + slots - 1) / slots;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    const int64_t units = M > 0 ? groups * parts : 0;
    return {per_gate, units, (int)parts, (int)(units < blocks ? units : blocks)};
}

static bool bad_pitch(int64_t ld, int64_t D) { return ld < D || (ld % 8); }

static f8_status check_residual(int64_t M, int64_t D, const void* gate, int64_t gate_rows, float a, float b)
{
    if (M < 0 || M > 0x7FFFFFFF || D < 0 || D > kRowMaxD || (D % 8) || gate_rows < 0 || gate_rows > 0x7FFFFFFF || gate_rows * D > 0x7FFFFFFFFLL ||
        (gate != nullptr) != (gate_rows > 0) || (gate_rows > 0 && M % gate_rows) || !(a - a == 0.0f) || !(b - b == 0.0f))
        return F8_ERR_SHAPE;
    return F8_OK;
}

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_residual_norm_bwd_workspace_bytes(int64_t M, int64_t D, int64_t gate_rows)
{
    if (check_residual(M, D, gate_rows > 0 ? &M : nullptr, gate_rows, 1.0f, 1.0f) != F8_OK) return kMinWorkspaceBytes;
    const ResidualPlan plan = plan_bwd(M, D, gate_rows);
    const size_t rows = (size_t)plan.blocks * 2 + (gate_rows > 0 && plan.parts > 1 ? (size_t)plan.units : 0);
    return kMinWorkspaceBytes + rows * D * sizeof(float);
}

f8_status f8_residual_norm(const void* x_bf16, int64_t ldx, const void* y_bf16, int64_t ldy, int64_t M, int64_t D, const void* g_post_bf16,
                           const void* gate_bf16, int64_t gate_rows, const void* g_pre_bf16, float skip_scale, float branch_scale, float eps,
                           void* h_bf16, int64_t ldh, void* n_bf16, int64_t ldn, float* rstd_post, float* rstd_pre, float* amax_n,
                           void* workspace, size_t workspace_bytes_, void* stream)
{
    if (M != 0 && (!x_bf16 || !y_bf16 || !h_bf16 || (n_bf16 != nullptr) != (g_pre_bf16 != nullptr) || (!g_post_bf16 && rstd_post) ||
                   (!g_pre_bf16 && (rstd_pre || amax_n))))
        return F8_ERR_NULL;  // (without rows there is nothing that these point to)
    f8_status s = check_residual(M, D, gate_bf16, gate_rows, skip_scale, branch_scale);
    if (s != F8_OK) return s;
    if (!(eps >= 0.0f) || bad_pitch(ldx, D) || bad_pitch(ldy, D) || bad_pitch(ldh, D) || (n_bf16 && bad_pitch(ldn, D))) return F8_ERR_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(y_bf16) || !aligned16(h_bf16) || !aligned16(n_bf16) || !aligned16(g_post_bf16) || !aligned16(gate_bf16) ||
        !aligned16(g_pre_bf16))
        return F8_ERR_ALIGN;
    if (amax_n && (!workspace || workspace_bytes_ < kMinWorkspaceBytes)) return F8_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    int nb = 0;
    if (M > 0 && D > 0) {
        const ResidualArgs a = {(const uint16_t*)x_bf16, (const uint16_t*)y_bf16, ldx, ldy, (const uint4*)g_post_bf16, (const uint4*)gate_bf16,
                                (const uint4*)g_pre_bf16, M, gate_rows > 0 ? M / gate_rows : M, (int)(D / 8), skip_scale, branch_scale, eps,
                                1.0f / (float)D, 1.0 / (double)D, (uint16_t*)h_bf16, (uint16_t*)n_bf16, ldh, ldn, rstd_post, rstd_pre,
                                amax_n ? (uint32_t*)workspace : nullptr};
        with_row_shape(D / 8, [&](auto T, auto U, int threads) {
            constexpr int kRows = T() == kWave ? kWaveRows : 1;
            const int64_t b = (M + kRows - 1) / kRows;
            nb = (int)(b < kResBlocks ? b : kResBlocks);
            const auto kernel = g_post_bf16 ? (g_pre_bf16 ? residual_norm_kernel<T(), U(), true, true> : residual_norm_kernel<T(), U(), true, false>)
                                            : (g_pre_bf16 ? residual_norm_kernel<T(), U(), false, true> : residual_norm_kernel<T(), U(), false, false>);
            kernel<<<nb, threads, 0, st>>>(a);
        });
    }
    if (amax_n) amax_final((const uint32_t*)workspace, nb, amax_n, st);
    return last_launch_status();
}

f8_status f8_residual_norm_bwd(const void* h_bf16, int64_t ldh, const void* y_bf16, int64_t ldy, const void* dh_bf16, int64_t lddh, const void* dn_bf16,
                               int64_t lddn, int64_t M, int64_t D, const void* g_post_bf16, const void* gate_bf16, int64_t gate_rows,
                               const void* g_pre_bf16, const float* rstd_post, const float* rstd_pre, float skip_scale, float branch_scale,
                               void* dx_bf16, int64_t lddx, void* dy_bf16, int64_t lddy, float* dg_post, float* dgate, float* dg_pre,
                               float* amax_dy, void* workspace, size_t workspace_bytes_, void* stream)
{
    const bool post = g_post_bf16, gated = gate_bf16, pre = g_pre_bf16;
    if (M != 0 && ((dn_bf16 != nullptr) != pre || (pre && (!h_bf16 || !rstd_pre)) || (!pre && !dh_bf16) || (post && !rstd_post) || ((post || gated) && !y_bf16) ||
        (dg_post && !post) || (dgate && !gated) || (dg_pre && !pre) || (amax_dy && !dy_bf16) || (!dx_bf16 && !dy_bf16 && !dg_post && !dgate && !dg_pre)))
        return F8_ERR_NULL;
    f8_status s = check_residual(M, D, gate_bf16, gate_rows, skip_scale, branch_scale);
    if (s != F8_OK) return s;
    if ((pre && (bad_pitch(ldh, D) || bad_pitch(lddn, D))) || ((post || gated) && bad_pitch(ldy, D)) || (dh_bf16 && bad_pitch(lddh, D)) ||
        (dx_bf16 && bad_pitch(lddx, D)) || (dy_bf16 && bad_pitch(lddy, D)))
        return F8_ERR_SHAPE;
    if (!aligned16(h_bf16) || !aligned16(y_bf16) || !aligned16(dh_bf16) || !aligned16(dn_bf16) || !aligned16(g_post_bf16) || !aligned16(gate_bf16) ||
        !aligned16(g_pre_bf16) || !aligned16(dx_bf16) || !aligned16(dy_bf16) || !aligned16(workspace))
        return F8_ERR_ALIGN;
    const ResidualPlan plan = plan_bwd(M, D, gate_rows);
    if ((dg_post || dgate || dg_pre || amax_dy) && (!workspace || workspace_bytes_ < f8_residual_norm_bwd_workspace_bytes(M, D, gate_rows))) return F8_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    uint32_t* const maxima = (uint32_t*)workspace;
    float* const sums = (float*)((char*)workspace + kMinWorkspaceBytes);
    const int64_t set = (int64_t)plan.blocks * D;
    const bool direct = plan.parts == 1;  // a unit is all rows of a gate row: its sum is the gradient
    if (M > 0 && D > 0) {
        const ResidualGradArgs a = {(const uint16_t*)h_bf16, (const uint16_t*)y_bf16, (const uint16_t*)dh_bf16, (const uint16_t*)dn_bf16, ldh, ldy, lddh, lddn,
                                    (const uint4*)g_post_bf16, (const uint4*)gate_bf16, (const uint4*)g_pre_bf16, rstd_post, rstd_pre, M, plan.per_gate,
                                    plan.units, plan.parts, (int)(D / 8), skip_scale, branch_scale, 1.0f / (float)D, (uint16_t*)dx_bf16, (uint16_t*)dy_bf16,
                                    lddx, lddy, dg_pre ? sums : nullptr, dg_post ? sums + set : nullptr,
                                    dgate ? (direct ? dgate : sums + 2 * set) : nullptr, amax_dy ? maxima : nullptr};
        with_bwd_shape(D / 8, [&](auto T, auto U, int threads) {
            const auto pick = [&](auto ONCE) {
                constexpr bool O = ONCE();
                return post ? (gated ? (pre ? residual_norm_bwd_kernel<T(), U(), true, true, true, O> : residual_norm_bwd_kernel<T(), U(), true, true, false, O>)
                                     : (pre ? residual_norm_bwd_kernel<T(), U(), true, false, true, O> : residual_norm_bwd_kernel<T(), U(), true, false, false, O>))
                            : (gated ? (pre ? residual_norm_bwd_kernel<T(), U(), false, true, true, O> : residual_norm_bwd_kernel<T(), U(), false, true, false, O>)
                                     : (pre ? residual_norm_bwd_kernel<T(), U(), false, false, true, O> : residual_norm_bwd_kernel<T(), U(), false, false, false, O>));
            };
            const auto kernel = M * D >= kResOnce ? pick(std::true_type{}) : pick(std::false_type{});
            kernel<<<plan.blocks, threads, 0, st>>>(a);
        });
    }
    ColumnSums f = {};
    if (dg_pre) f.part[f.sets] = sums, f.out[f.sets++] = dg_pre;
    if (dg_post) f.part[f.sets] = sums + set, f.out[f.sets++] = dg_post;
    f.strips = plan.blocks, f.parts = plan.parts, f.part_gate = sums + 2 * set, f.dgate = dgate, f.D = D;
    const int64_t gate_sets = dgate && !direct ? gate_rows : 0;  // (fewer than blocks)
    if (M == 0 && dgate && D > 0) {  // no rows: zeros
        ColumnSums z = {};
        z.dgate = dgate, z.D = gate_rows * D;
        column_sums(z, 1, st);
    }
    if (f.sets + gate_sets > 0 && D > 0) {
        if (amax_dy) f.partial = maxima, f.npartial = plan.blocks, f.amax = amax_dy;
        column_sums(f, (unsigned)(f.sets + gate_sets), st);
    } else if (amax_dy) {
        amax_final(maxima, D > 0 ? plan.blocks : 0, amax_dy, st);
    }
    return last_launch_status();
}

}  // extern "C"
