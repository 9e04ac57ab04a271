// Products of microscaled 4-bit operands, D[m, n] = bf16(sum over k of A[m, k] B[n, k]), on v_mfma_scale_f32_16x16x128_f8f6f4: a
// lane holds one block of 32 of one row (16 bytes of codes and a byte of scale), so the instruction applies the scales itself.
#include "f8_gemm_kernels.hpp"
#include "f8_mx4_device.hpp"

namespace f8 {

constexpr int kFp4 = 4;         // the instruction's format number
constexpr int kMxStep = 2 * kBK;  // elements of a step: rows of 128 bytes, two instructions

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
__device__ inline v8i fp4_operand(v4i x) { return v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}; }

__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p; }
__device__ inline v4u buffer_at(const uint8_t* p) { return v4u{(uint32_t)(uint64_t)p, (uint32_t)((uint64_t)p >> 32), kRecords, 0x00020000u}; }

// Few rows: tiles of 16 TM x 16 TN whose four waves take every fourth step each, through a ring of STAGES steps in LDS that is
// the wave's own, as in f8_gemm_rows.hip: no barrier until the sums meet, and the whole LDS is in flight.
template <int TM, int TN, int STAGES>
__global__ __launch_bounds__(256) void mx4_rows_kernel(const Mx4Args p, int tiles_m, int tiles_n)
{
    constexpr int NW = 4, ROWS = 16 * TM, COLS = 16 * TN, PITCH = COLS + 4, T = TM + TN;
    constexpr int DATA = T * 16 * kBK, STAGE = DATA + T * 256, LOADS = 3 * T;
    static_assert(NW * ROWS * PITCH * 4 <= NW * STAGES * STAGE && NW * STAGES * STAGE <= 160 * 1024 && (STAGES - 1) * LOADS < 64, "LDS; wait count");
    __shared__ __attribute__((aligned(1024))) uint8_t ring[NW][STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fr = lane & 15, fg = lane >> 4;
    int tm, tn;
    tile_coords((int)blockIdx.x, tiles_m, tiles_n, &tm, &tn);
    const int m0 = tm * ROWS, n0 = tn * COLS;
    const int64_t pitch = mx4_pitch(p.K);
    const uint8_t *a_base = p.A + m0 * pitch, *b_base = p.B + n0 * pitch;
    const int64_t a_scales = mx4_rows(p.M) * 16, b_scales = mx4_rows(p.N) * 16;  // bytes of a group
    const uint8_t *sa_base = p.sa + (int64_t)m0 * 16, *sb_base = p.sb + (int64_t)n0 * 16;

    // load l of a step: 8 rows of 128 bytes, A's rows first; lane: row lane / 8 of them, one 16-byte chunk.  Past the end of the
    // matrix or of the contraction it reads zeros.
    uint32_t off[2 * T];
    const int row8 = lane >> 3, chunk = 16 * ((lane & 7) ^ swz(row8));  // (the swizzle looks at bits 1 and 2 of the row only)
    static_for<2 * T>([&](auto L) {
        constexpr int l = L(), r = l < 2 * TM ? 8 * l : 8 * (l - 2 * TM);
        const int row = r + row8, left = l < 2 * TM ? p.M - m0 : p.N - n0;
        off[l] = row < left ? (uint32_t)row * (uint32_t)pitch + chunk : kPastEnd;
    });
    const uint32_t scale_off = fr * 16 + fg * 4;
    const int steps = (p.K + kMxStep - 1) / kMxStep;
    auto request = [&](int i, int stage) {  // step wave + 4 i
        const int kt = wave + NW * i, left = (int)(pitch - (int64_t)kt * kBK);  // bytes of a row from the step's first on; may be negative
        const int64_t at = kt < steps ? kt : 0;
        const v4u a = buffer_at(a_base + at * kBK), b = buffer_at(b_base + at * kBK);
        const v4u sa = buffer_at(sa_base + at / 2 * a_scales), sb = buffer_at(sb_base + at / 2 * b_scales);
        const uint32_t to = lds_address(ring[wave][stage]);
        static_for<2 * T>([&](auto L) {
            constexpr int l = L();
            const uint32_t o = chunk < left ? off[l] : kPastEnd, lds = to + l * 1024;
            const v4u src = l < 2 * TM ? a : b;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
        static_for<T>([&](auto L) {
            constexpr int l = L();
            const uint32_t o = kt < steps ? scale_off + (l < TM ? l : l - TM) * 256 : kPastEnd, lds = to + DATA + l * 256;
            const v4u src = l < TM ? sa : sb;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
    };
    v4f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    const int mine = (steps - wave + NW - 1) / NW;
    static_for<STAGES - 1>([&](auto I) { request(I(), I()); });
    constexpr int kWait = (STAGES - 2) * LOADS;
    int stage = 0;
    for (int i = 0; i < mine; ++i) {
        // the oldest step has landed; this wave's reads of the step before it are done, whose place the request takes
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kWait) : "memory");
        request(i + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        const uint8_t* st = ring[wave][stage];
        // a group's word holds four instructions' scales: the odd steps' are its upper half
        int scale[T];
#pragma unroll
        for (int x = 0; x < T; ++x) scale[x] = *reinterpret_cast<const int*>(st + DATA + x * 256 + lane * 4) >> 16 * (wave & 1);
        static_for<2>([&](auto J) {
            constexpr int j = J();
            v8i f[T];
#pragma unroll
            for (int x = 0; x < T; ++x) f[x] = fp4_operand(*reinterpret_cast<const v4i*>(st + (16 * x + fr) * kBK + 16 * ((4 * j + fg) ^ swz(fr))));
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f[TM + y], f[x], acc[x][y], kFp4, kFp4, j, scale[TM + y], j, scale[x]);
        });
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may still be writing the ring
    __syncthreads();
    float(*sums)[ROWS][PITCH] = reinterpret_cast<float(*)[ROWS][PITCH]>(&ring[0][0][0]);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<v4f*>(&sums[wave][16 * i + fr][16 * j + 4 * fg]) = acc[i][j];
    __syncthreads();
    for (int q = threadIdx.x; q < ROWS * COLS / 4; q += 256) {  // four neighbouring outputs
        const int r = q / (COLS / 4), c = q % (COLS / 4) * 4, m = m0 + r, n = n0 + c;
        if (m >= p.M || n >= p.N) continue;
        v4f t = *reinterpret_cast<const v4f*>(&sums[0][r][c]);
#pragma unroll
        for (int w = 1; w < NW; ++w) t += *reinterpret_cast<const v4f*>(&sums[w][r][c]);
        *reinterpret_cast<uint2*>(p.D + (int64_t)m * p.ldd + n) = make_uint2(pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3]));
    }
}

// ---- host ----------------------------------------------------------------------------------------

template <int TM, int TN, int STAGES>
static void launch_rows(const Mx4Args& a, hipStream_t st)
{
    const int tiles_m = (a.M + 16 * TM - 1) / (16 * TM), tiles_n = (a.N + 16 * TN - 1) / (16 * TN);
    mx4_rows_kernel<TM, TN, STAGES><<<(unsigned)(tiles_m * tiles_n), 256, 0, st>>>(a, tiles_m, tiles_n);
}

size_t mx4_split_bytes(int64_t, int64_t, int64_t) { return 0; }

f8_status mx4_gemm(const Mx4Args& a, void*, size_t, hipStream_t st)
{
    if (a.M == 0 || a.N == 0) return last_launch_status();
    if (a.M <= 16) launch_rows<1, 2, 5>(a, st);
    else if (a.M <= 32) launch_rows<2, 2, 4>(a, st);
    else launch_rows<4, 4, 2>(a, st);
    return last_launch_status();
}

}  // namespace f8
