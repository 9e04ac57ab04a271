// Layer norm, alone or behind a residual sum, forward and backward:
//   h = bf16(x + y) (or x),  mean = sum h / D,  rstd = 1 / sqrt(sum (h - mean)^2 / D + eps),  n = (h - mean) rstd g + b;
//   with c = (h - mean) rstd and v = g dn:  dx = rstd (v - mean(v) - c mean(v c)) + dh,  dg = sum dn c,  db = sum dn.
// Bound by memory: 4 bytes an element forward (8 with the sum), 6 backward (8 with the sum's gradient).  A row is held in
// registers, so that the mean, the sum of squares around it and the result take one reading; both gains' sums run along in the
// backward's one pass and are joined over the blocks by a second launch, in a fixed order.
// The mean is held in fp32, also for the backward: of r deviations, its rounding moves the differences by 2^-24 r deviations.
// 16384 x 8192 with a residual, us: forward 181 to 185, backward 177 to 200 (5.8 and 5.4 to 6.0 TB/s; a large copy 5.0); 8192 x 4096
// 40.5 to 53 (53 over sets of inputs that no cache holds) and 50; 2001 x 2816 without 7 and 16.
#include "f8_rows.hpp"

namespace f8 {

constexpr int kLnBlocks = 2048;  // of the forward with a maximum over n: one partial maximum each
static_assert((size_t)kLnBlocks * sizeof(uint32_t) <= kMinWorkspaceBytes, "one partial per block fits the minimum workspace");
constexpr int kLnBwdBlocks = 512;  // of the backward at most, each of which leaves a partial row of both sums
constexpr int64_t kLnOnce = (int64_t)1 << 25;  // elements from which the backward loads past the caches

struct LayerNormArgs {
    const uint16_t *x, *y;
    int64_t ldx, ldy;
    const uint4 *g, *b;  // b nullable
    int64_t M;
    int dc;  // 16-byte chunks of a row
    float eps;
    double inv_d;
    uint16_t *h, *n;
    int64_t ldh, ldn;
    float *mean, *rstd;
    uint32_t* partial;
};

// Sums of two numbers over the threads of a row.  Two buffers in turn and one barrier: a buffer is written again only after the
// barrier of the sum in between.
template <int THREADS>
struct RowSums {
    float2 (*part)[16];
    int buf = 0;
    __device__ float2 operator()(float2 v)
    {
        const auto add = [](float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); };
        v = wave_all(v, add);
        if constexpr (THREADS > kWave) {
            const int waves = blockDim.x / kWave;
            if (threadIdx.x % kWave == 0) part[buf][threadIdx.x / kWave] = v;
            __syncthreads();
            v = part[buf][0];
            for (int w = 1; w < waves; ++w) v = add(v, part[buf][w]);
            buf ^= 1;
        }
        return v;
    }
};

template <int THREADS, int U, bool SUM>
__global__ __launch_bounds__(block_threads(THREADS)) void layernorm_kernel(const LayerNormArgs p)
{
    constexpr int kRows = THREADS == kWave ? kWaveRows : 1;
    __shared__ float2 part[2][16];
    __shared__ uint32_t red[block_threads(THREADS) / kWave];
    RowSums<THREADS> sums{part};
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
            if (in[u]) x[u] = row_of(p.x, m, p.ldx)[c];
            if (SUM && in[u]) y[u] = row_of(p.y, m, p.ldy)[c];
        }
        float f[U][8], s = 0.0f, q = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unpack8(x[u], f[u]);
            if constexpr (SUM) {
                float fy[8];
                unpack8(y[u], fy);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[u][j] += fy[j];
                const uint4 h = pack8(f[u]);
                if (in[u]) row_of(p.h, m, p.ldh)[t + TPR * u] = h;
                unpack8(h, f[u]);  // the norm is that of the sum that is kept
            }
            s += ((f[u][0] + f[u][1]) + (f[u][2] + f[u][3])) + ((f[u][4] + f[u][5]) + (f[u][6] + f[u][7]));
        }
        const float mean = (float)((double)sums(make_float2(s, 0.0f)).x * p.inv_d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[u][j] -= mean, d[j] = f[u][j] * f[u][j];
            if (in[u]) q += ((d[0] + d[1]) + (d[2] + d[3])) + ((d[4] + d[5]) + (d[6] + d[7]));
        }
        const float rstd = rsqrt_exact((double)sums(make_float2(q, 0.0f)).x * p.inv_d + (double)p.eps);
        if (t == 0 && live) {
            if (p.mean) p.mean[m] = mean;
            if (p.rstd) p.rstd[m] = rstd;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            const int c = t + TPR * u;
            float g[8], b[8];
            unpack8(p.g[c], g);
            if (p.b) unpack8(p.b[c], b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[u][j] = (f[u][j] * rstd) * g[j];
                if (p.b) f[u][j] += b[j];
            }
            const uint4 o = pack8(f[u]);
            row_of(p.n, m, p.ldn)[c] = o;
            mag = absmax_acc(mag, o);
        }
    }
    if (p.partial) {
        const uint32_t mx = waves_max(pk_collapse(mag), red);
        if (threadIdx.x == 0) p.partial[blockIdx.x] = mx;
    }
}

// ---- backward ----------------------------------------------------------------------------------

struct LayerNormGradArgs {
    const uint16_t *h, *dn, *dh;  // dh nullable
    int64_t ldh, lddn, lddh;
    const uint4* g;
    const float *mean, *rstd;
    int64_t M;
    int dc;
    float inv_d;
    uint16_t* dx;  // nullable
    int64_t lddx;
    float *part_g, *part_b;  // nullable, [block][D]
    uint32_t* partial;
};

// Block b takes the rows b * kRows, ... of every gridDim.x * kRows.
template <int THREADS, int U, bool ONCE>
__global__ __launch_bounds__(block_threads(THREADS)) void layernorm_bwd_kernel(const LayerNormGradArgs p)
{
    constexpr int kRows = THREADS == kWave ? kWaveRows : 1;
    __shared__ float2 part[2][16];
    __shared__ float share[kRows][kRows > 1 ? kWave * U * 8 : 1];
    __shared__ uint32_t red[block_threads(THREADS) / kWave];
    RowSums<THREADS> sums{part};
    const int TPR = THREADS == kWave ? kWave : (int)blockDim.x;
    const int t = THREADS == kWave ? (int)threadIdx.x % kWave : (int)threadIdx.x, sub = THREADS == kWave ? (int)threadIdx.x / kWave : 0;
    uint32_t mag = 0;
    float acc_g[U][8] = {}, acc_b[U][8] = {};
    uint4 gain[U];
#pragma unroll
    for (int u = 0; u < U; ++u) gain[u] = t + TPR * u < p.dc ? p.g[t + TPR * u] : make_uint4(0, 0, 0, 0);
    struct Row {
        uint4 h[U], dn[U], dh[U];
        float mean, rstd;
    };
    const int64_t stride = (int64_t)gridDim.x * kRows;
    const auto load_row = [&](Row& row, int64_t m) {
        const bool live = m < p.M;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            row.h[u] = row.dn[u] = row.dh[u] = make_uint4(0, 0, 0, 0);
            if (!live || c >= p.dc) continue;
            const auto load = [&](const uint16_t* a, int64_t ld) { return ONCE ? load_once(row_of(a, m, ld) + c) : row_of(a, m, ld)[c]; };
            row.h[u] = load(p.h, p.ldh), row.dn[u] = load(p.dn, p.lddn);
            if (p.dh && p.dx) row.dh[u] = load(p.dh, p.lddh);
        }
        row.mean = live ? p.mean[m] : 0.0f, row.rstd = live ? p.rstd[m] : 0.0f;
    };
    Row next;
    load_row(next, (int64_t)blockIdx.x * kRows + sub);
    for (int64_t m0 = (int64_t)blockIdx.x * kRows; m0 < p.M; m0 += stride) {
        const int64_t m = m0 + sub;
        const bool live = m < p.M;
        const Row row = next;
        load_row(next, m + stride);
        const uint4(&h)[U] = row.h;
        const uint4(&dn)[U] = row.dn;
        const uint4(&dh)[U] = row.dh;
        const float mean = row.mean, rstd = row.rstd;
        float2 s = make_float2(0.0f, 0.0f);
        // (past the row's end dn and the gain are zero, and so is every term)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float fh[8], fd[8], g[8], a[8];
            unpack8(h[u], fh), unpack8(dn[u], fd), unpack8(gain[u], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = (fh[j] - mean) * rstd;
                acc_g[u][j] += fd[j] * c;
                acc_b[u][j] += fd[j];
                g[j] *= fd[j];
                a[j] = g[j] * c;
            }
            s.x += ((g[0] + g[1]) + (g[2] + g[3])) + ((g[4] + g[5]) + (g[6] + g[7]));
            s.y += ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
        }
        if (!p.dx) continue;  // uniform
        s = sums(s);
        const float mv = s.x * p.inv_d, mvc = s.y * p.inv_d;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            float fh[8], fd[8], g[8], fa[8];
            unpack8(h[u], fh), unpack8(dn[u], fd), unpack8(gain[u], g), unpack8(dh[u], fa);
#pragma unroll
            for (int j = 0; j < 8; ++j) fa[j] += rstd * ((g[j] * fd[j] - mv) - ((fh[j] - mean) * rstd) * mvc);
            const uint4 o = pack8(fa);
            if (live && c < p.dc) {
                store_stream(row_of(p.dx, m, p.lddx) + c, o);
                mag = absmax_acc(mag, o);
            }
        }
    }
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
                    float v = share[0][(u * 8 + j) * kWave + t];
                    for (int k = 1; k < kRows; ++k) v += share[k][(u * 8 + j) * kWave + t];
                    acc[u][j] = v;
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = t + TPR * u;
            if (c >= p.dc) continue;
            float4* o = reinterpret_cast<float4*>(out + (int64_t)c * 8);
            o[0] = make_float4(acc[u][0], acc[u][1], acc[u][2], acc[u][3]), o[1] = make_float4(acc[u][4], acc[u][5], acc[u][6], acc[u][7]);
        }
    };
    if (p.part_g) leave(acc_g, p.part_g + (int64_t)blockIdx.x * p.dc * 8);
    if (p.part_b) leave(acc_b, p.part_b + (int64_t)blockIdx.x * p.dc * 8);
    if (p.partial) {
        const uint32_t mx = waves_max(pk_collapse(mag), red);
        if (threadIdx.x == 0) p.partial[blockIdx.x] = mx;
    }
}

// ---- host ----------------------------------------------------------------------------------------

template <class F>
static void with_grad_shape(int64_t dc, F&& f)
{
    if (dc <= 64) f(Threads<64>{}, One{}, block_threads(64));
    else if (dc <= 128) f(Threads<64>{}, Two{}, block_threads(64));
    else if (dc <= 1024) with_block(dc, One{}, f);
    else f(Threads<1024>{}, Two{}, (int)((dc + 2 * kWave - 1) / (2 * kWave)) * kWave);
}

static int bwd_blocks(int64_t M, int64_t D)
{
    const int64_t slots = D / 8 <= 128 ? kWaveRows : 1, most = (M + slots - 1) / slots;
    // Rows of seven waves and more: half as many, as few loads at a time are enough then and partial rows cost (8192 x 4096 49.6 us for
    // 54.6, 300 x 4096 11.3 for 12.6, 16384 x 3584 82.5 for 84, 1000 x 8192 21.2 for 28.5; but 32768 x 2816 139 for 127, 16384 x 2048 63
    // for 51).
    const int blocks = D / 8 > 6 * kWave ? kLnBwdBlocks / 2 : kLnBwdBlocks;
    return (int)(most < blocks ? most : blocks);
}

static bool bad_size(int64_t M, int64_t D) { return M < 0 || M > 0x7FFFFFFF || D < 0 || D > kRowMaxD || (D % 8); }
static bool bad_pitch(int64_t ld, int64_t D) { return ld < D || (ld % 8); }

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_layernorm_bwd_workspace_bytes(int64_t M, int64_t D)
{
    if (bad_size(M, D)) return kMinWorkspaceBytes;
    return kMinWorkspaceBytes + (size_t)bwd_blocks(M, D) * 2 * D * sizeof(float);
}

f8_status f8_layernorm(const void* x_bf16, int64_t ldx, const void* y_bf16, int64_t ldy, int64_t M, int64_t D, const void* g_bf16,
                       const void* b_bf16, float eps, void* h_bf16, int64_t ldh, void* n_bf16, int64_t ldn, float* mean, float* rstd,
                       float* amax_n, void* workspace, size_t workspace_bytes_, void* stream)
{
    if (bad_size(M, D) || !(eps >= 0.0f) || !(eps - eps == 0.0f)) return F8_ERR_SHAPE;
    if (!g_bf16 || (M != 0 && (!x_bf16 || !n_bf16 || (y_bf16 != nullptr) != (h_bf16 != nullptr)))) return F8_ERR_NULL;
    if (bad_pitch(ldx, D) || bad_pitch(ldn, D) || (y_bf16 && (bad_pitch(ldy, D) || bad_pitch(ldh, D)))) return F8_ERR_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(y_bf16) || !aligned16(g_bf16) || !aligned16(b_bf16) || !aligned16(h_bf16) || !aligned16(n_bf16)) return F8_ERR_ALIGN;
    if (amax_n && (!workspace || workspace_bytes_ < kMinWorkspaceBytes)) return F8_ERR_WORKSPACE;
    if (amax_n && !aligned16(workspace)) return F8_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    int nb = 0;
    if (M > 0 && D > 0) {
        const LayerNormArgs a = {(const uint16_t*)x_bf16, (const uint16_t*)y_bf16, ldx, ldy, (const uint4*)g_bf16, (const uint4*)b_bf16, M, (int)(D / 8), eps,
                                 1.0 / (double)D, (uint16_t*)h_bf16, (uint16_t*)n_bf16, ldh, ldn, mean, rstd, amax_n ? (uint32_t*)workspace : nullptr};
        with_row_shape(D / 8, [&](auto T, auto U, int threads) {
            constexpr int kRows = T() == kWave ? kWaveRows : 1;
            const int64_t b = (M + kRows - 1) / kRows;
            // rows in the order of the blocks' start read and write faster than rows at a stride of the grid (16384 x 8192 with a
            // residual 184 us for 198, 8192 x 4096 40.7 for 43); where each block leaves a maximum, there is room for so many
            // (with the launch that joins the maxima 202 us for 185, 8192 x 4096 56 for 53, 2001 x 2816 without a residual 11.4 for 7.2)
            const int64_t most = amax_n ? kLnBlocks : 0x7FFFFFFF / threads;
            nb = (int)(b < most ? b : most);
            const auto kernel = y_bf16 ? layernorm_kernel<T(), U(), true> : layernorm_kernel<T(), U(), false>;
            kernel<<<nb, threads, 0, st>>>(a);
        });
    }
    if (amax_n) amax_final((const uint32_t*)workspace, nb, amax_n, st);
    return last_launch_status();
}

f8_status f8_layernorm_bwd(const void* h_bf16, int64_t ldh, const void* g_bf16, const float* mean, const float* rstd, const void* dn_bf16, int64_t lddn,
                           const void* dh_bf16, int64_t lddh, int64_t M, int64_t D, void* dx_bf16, int64_t lddx, float* dg, float* db, float* amax_dx,
                           void* workspace, size_t workspace_bytes_, void* stream)
{
    if (bad_size(M, D)) return F8_ERR_SHAPE;
    if (!g_bf16 || (M != 0 && (!h_bf16 || !mean || !rstd || !dn_bf16 || (!dx_bf16 && (dh_bf16 || amax_dx)))) || (!dx_bf16 && !dg && !db)) return F8_ERR_NULL;
    if (bad_pitch(ldh, D) || bad_pitch(lddn, D) || (dh_bf16 && bad_pitch(lddh, D)) || (dx_bf16 && bad_pitch(lddx, D))) return F8_ERR_SHAPE;
    if (!aligned16(h_bf16) || !aligned16(g_bf16) || !aligned16(dn_bf16) || !aligned16(dh_bf16) || !aligned16(dx_bf16) || !aligned16(workspace)) return F8_ERR_ALIGN;
    if ((dg || db || amax_dx) && (!workspace || workspace_bytes_ < f8_layernorm_bwd_workspace_bytes(M, D))) return F8_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int blocks = bwd_blocks(M, D);
    uint32_t* const maxima = (uint32_t*)workspace;
    float* const sums = (float*)((char*)workspace + kMinWorkspaceBytes);
    const int64_t set = (int64_t)blocks * D;
    if (M > 0 && D > 0) {
        const LayerNormGradArgs a = {(const uint16_t*)h_bf16, (const uint16_t*)dn_bf16, (const uint16_t*)dh_bf16, ldh, lddn, lddh, (const uint4*)g_bf16, mean, rstd, M,
                                     (int)(D / 8), 1.0f / (float)D, (uint16_t*)dx_bf16, lddx, dg ? sums : nullptr, db ? sums + set : nullptr, amax_dx ? maxima : nullptr};
        with_grad_shape(D / 8, [&](auto T, auto U, int threads) {
            const auto kernel = M * D >= kLnOnce ? layernorm_bwd_kernel<T(), U(), true> : layernorm_bwd_kernel<T(), U(), false>;
            kernel<<<blocks, threads, 0, st>>>(a);
        });
    }
    ColumnSums f = {};
    if (dg) f.part[f.sets] = sums, f.out[f.sets++] = dg;
    if (db) f.part[f.sets] = sums + set, f.out[f.sets++] = db;
    f.strips = blocks, f.D = D;
    if (f.sets > 0 && D > 0) {
        if (amax_dx) f.partial = maxima, f.npartial = blocks, f.amax = amax_dx;
        column_sums(f, (unsigned)f.sets, st);
    } else if (amax_dx) {
        amax_final(maxima, D > 0 ? blocks : 0, amax_dx, st);
    }
    return last_launch_status();
}

}  // extern "C"
