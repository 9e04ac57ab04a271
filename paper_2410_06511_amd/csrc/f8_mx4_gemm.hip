// Products of microscaled 4-bit operands, D[m, n] = bf16(sum over k of A[m, k] B[n, k]), on v_mfma_scale_f32_16x16x128_f8f6f4: a
// lane holds one block of 32 of one row (16 bytes of codes and a byte of scale), so the instruction applies the scales itself.
#include "f8_gemm_kernels.hpp"
#include "f8_mx4_device.hpp"

namespace f8 {

constexpr int kFp4 = 4;         // the instruction's format number
constexpr int kMxStep = 2 * kBK;  // elements of a step: rows of 128 bytes, two instructions

// Order of a row's eight 16-byte chunks in LDS: chunk c at c ^ mx4_swz(row).  A lane of an operand reads chunk fg or 4 + fg of row fr,
// where the 8-bit products read 2 fg and 2 fg + 1, and their order costs conflicts here: 8192 x 4096 x 14336 183 us for 179, 300 x 4096
// x 4096 10.3 for 9.9 (row & 6 as good to 0.5 %, row >> 1 & 3 as theirs).
__device__ inline int mx4_swz(int row) { return row & 7; }

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
// (an fp4 operand is four registers; what the builtin's type has above them is never read)
__device__ inline v8i fp4_operand(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p; }
__device__ inline v4u buffer_at(const uint8_t* p) { return v4u{(uint32_t)(uint64_t)p, (uint32_t)((uint64_t)p >> 32), kRecords, 0x00020000u}; }

// Few rows: tiles of 16 TM x 16 TN whose four waves take every fourth step each, through a ring of STAGES steps in LDS that is
// the wave's own, as in f8_gemm_rows.hip: no barrier until the sums meet, and the whole LDS is in flight.
// TOKENS (TM = 1): A comes as up to kMxTokens rows of bf16, which every workgroup quantises for itself while its first steps of B
// are under way: the codes that mx4_cast_kernel would have written, in LDS and without its launch.  (A lane that quantises its own
// block in every step, on its way to the instruction, takes 0.8 us a step for it.)
template <int TM, int TN, int STAGES, bool TOKENS = false>
__global__ __launch_bounds__(256) void mx4_rows_kernel(const Mx4Args p, int tiles_m, int tiles_n, const uint16_t* __restrict__ X)
{
    static_assert(TM == 1 || !TOKENS, "");
    constexpr int NW = 4, ROWS = 16 * TM, COLS = 16 * TN, PITCH = COLS + 4, TA = TOKENS ? 0 : TM, T = TA + TN;  // fragments that come as codes
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
    const int64_t a_scales = p.a_srows * 16, b_scales = p.b_srows * 16;  // bytes of a group
    const uint8_t *sa_base = p.sa + (int64_t)m0 * 16, *sb_base = p.sb + (int64_t)n0 * 16;

    // load l of a step: 8 rows of 128 bytes, A's rows first; lane: row lane / 8 of them, one 16-byte chunk.  Past the end of the
    // matrix or of the contraction it reads zeros.
    uint32_t off[2 * T];
    const int row8 = lane >> 3, chunk = 16 * ((lane & 7) ^ mx4_swz(row8));
    static_for<2 * T>([&](auto L) {
        constexpr int l = L(), r = l < 2 * TA ? 8 * l : 8 * (l - 2 * TA);
        const int row = r + row8, left = l < 2 * TA ? p.M - m0 : p.N - n0;
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
            const v4u src = l < 2 * TA ? a : b;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
        static_for<T>([&](auto L) {
            constexpr int l = L();
            const uint32_t o = kt < steps ? scale_off + (l < TA ? l : l - TA) * 256 : kPastEnd, lds = to + DATA + l * 256;
            const v4u src = l < TA ? sa : sb;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
    };
    v4f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    const int mine = (steps - wave + NW - 1) / NW;
    extern __shared__ __attribute__((aligned(16))) uint8_t tokens[];  // TOKENS: codes [M][pitch], then scales [group][M][16]
    uint8_t* const token_scales = tokens + p.M * (int)pitch;
    const int words = (int)pitch / 4, all_words = p.M * words;  // of eight codes
    constexpr int FIRST = 2;
    uint4 x[FIRST];
    const auto eight = [&](int i) {  // the values of word i
        const int row = i / words, k = i % words * 8;
        return i < all_words && k < p.K ? *reinterpret_cast<const uint4*>(X + (int64_t)row * p.K + k) : make_uint4(0, 0, 0, 0);
    };
    const auto quantise = [&](int i, const uint4& v) {  // (four neighbouring lanes have a block)
        const uint32_t code = mx4_scale_of_quad(v);
        if (i >= all_words) return;
        const int row = i / words, k = i % words, b = k / 4;
        *reinterpret_cast<uint32_t*>(tokens + 4 * i) = mx4_encode8(v, code);
        if (k % 4 == 0) token_scales[(b / 16 * p.M + row) * 16 + 4 * (b % 4) + b % 16 / 4] = (uint8_t)code;
    };
    if constexpr (TOKENS) {
#pragma unroll
        for (int u = 0; u < FIRST; ++u) x[u] = eight(u * 256 + (int)threadIdx.x);
    }
    static_for<STAGES - 1>([&](auto I) { request(I(), I()); });
    if constexpr (TOKENS) {
#pragma unroll
        for (int u = 0; u < FIRST; ++u) quantise(u * 256 + (int)threadIdx.x, x[u]);
        for (int i0 = FIRST * 256; i0 < all_words; i0 += 4 * 256) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = eight(i0 + u * 256 + (int)threadIdx.x);
#pragma unroll
            for (int u = 0; u < 4; ++u) quantise(i0 + u * 256 + (int)threadIdx.x, v[u]);
        }
        __syncthreads();
    }
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
            v8i f[TM + TN];
            int sa[TM];
#pragma unroll
            for (int x = 0; x < T; ++x)
                f[TM - TA + x] = fp4_operand(*reinterpret_cast<const v4i*>(st + (16 * x + fr) * kBK + 16 * ((4 * j + fg) ^ mx4_swz(fr))));
            if constexpr (TOKENS) {
                const int kt = wave + NW * i;
                const bool some = fr < p.M && kt * kBK + 64 * j + 16 * fg < pitch;
                v4i codes = {0, 0, 0, 0};
                int word = 0;
                if (some) {
                    codes = *reinterpret_cast<const v4i*>(tokens + fr * (int)pitch + kt * kBK + 64 * j + 16 * fg);
                    word = *reinterpret_cast<const int*>(token_scales + (kt / 2 * p.M + fr) * 16 + 4 * fg);
                }
                f[0] = fp4_operand(codes);
                sa[0] = word >> 16 * (wave & 1);
            } else {
#pragma unroll
                for (int x = 0; x < TM; ++x) sa[x] = scale[x];
            }
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f[TM + y], f[x], acc[x][y], kFp4, kFp4, j, scale[TA + y], j, sa[x]);
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

// ---- few rows, many columns ------------------------------------------------------------------------

// Tiles of 16 TM x 64 with one ring of STAGES groups (512 elements of each row, with their scales) for eight waves: whatever the
// height of the tile, all of the LDS but one group is under way, with one barrier a group.  Wave w has all rows and 32 of the
// columns, and of each group the quarter w % 4; the four quarters' sums meet in LDS at the end.  (With 16 columns and half of each
// group a wave would read A twice as often; mx4_rows_kernel has a ring for each wave, which a tile of this size leaves two steps.)
// 300 x 4096 x 4096 9.9 us (1.0 PFLOP/s), 300 x 14336 x 4096 19.7: a unit's ring of 110 KB takes 2.3 us to come.
template <int TM, int STAGES>
__global__ __launch_bounds__(512) void mx4_strip_kernel(const Mx4Args p, int tiles_m, int tiles_n)
{
    constexpr int ROWS = 16 * TM, COLS = 64, HALF = (ROWS + COLS) * kBK, A_BYTES = ROWS * kBK, STAGE = 2 * HALF + (TM + 4) * 256;
    // loads of a wave and group: eight rows of 128 bytes each of A and B, 16 rows' scales
    constexpr int A_LOADS = TM / 2, B_LOADS = 2, S_LOADS = (TM + 4 + 7) / 8, LOADS = A_LOADS + B_LOADS + S_LOADS;
    constexpr int PITCH = COLS + 4;  // floats
    static_assert(TM % 2 == 0 && STAGES * STAGE <= 160 * 1024 && (STAGES - 1) * LOADS < 64 && 4 * ROWS * PITCH * 4 <= STAGES * STAGE, "LDS; wait count; the sums take the ring's place");
    __shared__ __attribute__((aligned(1024))) uint8_t ring[STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = wave % 4, cols0 = wave / 4 * 32, fr = lane & 15, fg = lane >> 4;
    int tm, tn;
    tile_coords((int)blockIdx.x, tiles_m, tiles_n, &tm, &tn);
    const int m0 = tm * ROWS, n0 = tn * COLS;
    const int64_t pitch = mx4_pitch(p.K);
    const uint8_t *a_base = p.A + m0 * pitch, *b_base = p.B + n0 * pitch;

    // Piece x of A: 8 rows (see mx4_rows_kernel) of the half x / (2 TM); wave w has the pieces w, w + 8, ..., of B the piece w of both
    // halves, of the scales (16 rows, A's first) w and w + 8, or the last one again.
    const int row8 = lane >> 3, chunk = 16 * ((lane & 7) ^ mx4_swz(row8));
    uint32_t a_off[A_LOADS], b_off, a_lds[A_LOADS], s_lds[S_LOADS];
    int a_begin[A_LOADS];  // of a lane's 16 bytes in a group's 256 of a row
    const uint8_t* s_base[S_LOADS];
    int64_t s_step[S_LOADS];
#pragma unroll
    for (int j = 0; j < A_LOADS; ++j) {
        const int x = wave + 8 * j, h = x / (2 * TM), y = x % (2 * TM), row = 8 * y + row8;
        a_begin[j] = h * kBK + chunk;
        a_off[j] = row < p.M - m0 ? (uint32_t)row * (uint32_t)pitch + a_begin[j] : kPastEnd;
        a_lds[j] = h * HALF + y * 1024;
    }
    b_off = 8 * wave + row8 < p.N - n0 ? (uint32_t)(8 * wave + row8) * (uint32_t)pitch + chunk : kPastEnd;
#pragma unroll
    for (int j = 0; j < S_LOADS; ++j) {
        const int x = wave + 8 * j < TM + 4 ? wave + 8 * j : TM + 3;
        const bool is_a = x < TM;
        const int64_t rows = is_a ? p.a_srows : p.b_srows, row = is_a ? m0 + 16 * x : n0 + 16 * (x - TM);
        s_base[j] = (is_a ? p.sa : p.sb) + (row < rows ? row : rows - 16) * 16;  // (past the end: some others)
        s_step[j] = rows * 16, s_lds[j] = 2 * HALF + x * 256;
    }
    const uint32_t scale_off = lane * 4;
    const int groups = (p.K + kMxGroup - 1) / kMxGroup;
    const uint32_t ring0 = lds_address(&ring[0][0]);
    auto request = [&](int g, int stage) {
        const int64_t left = pitch - (int64_t)g * 2 * kBK, at = g < groups ? g : 0;  // left: bytes of a row, may be negative
        const v4u a = buffer_at(a_base + at * 2 * kBK), b = buffer_at(b_base + at * 2 * kBK);
        const uint32_t to = ring0 + stage * STAGE;
        static_for<A_LOADS + B_LOADS>([&](auto J) {
            constexpr int j = J(), h = j - A_LOADS;
            uint32_t o, lds;
            if constexpr (j < A_LOADS) o = a_begin[j] < left ? a_off[j] : kPastEnd, lds = to + a_lds[j];
            else o = h * kBK + chunk < left ? b_off + h * kBK : kPastEnd, lds = to + h * HALF + A_BYTES + wave * 1024;
            const v4u src = j < A_LOADS ? a : b;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
        static_for<S_LOADS>([&](auto J) {
            const v4u src = buffer_at(s_base[J()] + at * s_step[J()]);
            const uint32_t o = g < groups ? scale_off : kPastEnd, lds = to + s_lds[J()];
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        });
    };
    v4f acc[TM][2];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i][0] = acc[i][1] = v4f{0.f, 0.f, 0.f, 0.f};
    static_for<STAGES - 1>([&](auto I) { request(I(), I()); });
    constexpr int kWait = (STAGES - 2) * LOADS;
    const int at = quarter / 2 * HALF + fr * kBK + 16 * ((quarter % 2 * 4 + fg) ^ mx4_swz(fr));  // of a fragment's first rows in a stage
    int stage = 0;
    for (int g = 0; g < groups; ++g) {
        // this wave's loads of the oldest group have landed, and behind the barrier everyone's; everyone is done with the group
        // before, whose place the request takes
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kWait) : "memory");
        request(g + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        const uint8_t *st = ring[stage] + at, *sc = ring[stage] + 2 * HALF + fr * 16 + fg * 4;
        v4i a[TM], b[2];
        int sa[TM], sb[2];  // (a word holds the four quarters' scales)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            b[j] = *reinterpret_cast<const v4i*>(st + A_BYTES + (cols0 + 16 * j) * kBK);
            sb[j] = *reinterpret_cast<const int*>(sc + (TM + cols0 / 16 + j) * 256) >> 8 * quarter;
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            a[i] = *reinterpret_cast<const v4i*>(st + 16 * i * kBK);
            sa[i] = *reinterpret_cast<const int*>(sc + i * 256) >> 8 * quarter;
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(b[j]), fp4_operand(a[i]), acc[i][j], kFp4, kFp4, 0, sb[j], 0, sa[i]);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no load may still be writing the ring
    __syncthreads();
    float(*sums)[ROWS][PITCH] = reinterpret_cast<float(*)[ROWS][PITCH]>(&ring[0][0]);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *reinterpret_cast<v4f*>(&sums[quarter][16 * i + fr][cols0 + 16 * j + 4 * fg]) = acc[i][j];
    __syncthreads();
    for (int q = threadIdx.x; q < ROWS * 8; q += 512) {  // eight neighbouring results
        const int r = q / 8, c = q % 8 * 8;
        if (m0 + r >= p.M || n0 + c >= p.N) continue;
        v4f lo = *reinterpret_cast<const v4f*>(&sums[0][r][c]), hi = *reinterpret_cast<const v4f*>(&sums[0][r][c + 4]);
#pragma unroll
        for (int k = 1; k < 4; ++k) lo += *reinterpret_cast<const v4f*>(&sums[k][r][c]), hi += *reinterpret_cast<const v4f*>(&sums[k][r][c + 4]);
        *reinterpret_cast<uint4*>(p.D + (int64_t)(m0 + r) * p.ldd + n0 + c) =
            make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
    }
}

// ---- tiles ---------------------------------------------------------------------------------------

// As gemm_tile_kernel (f8_gemm_kernels.hpp) for two operands whose contraction is contiguous: persistent workgroups, two LDS
// stages of 128 bytes of each row (256 elements here: two instructions of 128), loads two steps ahead of the products and spread
// over them, the same order of fragments.  What is different:
//   - a slot of the step, which there is one instruction of 32 cycles, is two of 16; the two of one accumulator are a slot apart.
//   - the scales of a pair of steps, 16 bytes for each row, come to LDS in the pair before and to registers in its last half step:
//     a word for each fragment, whose byte the instruction picks.
//   - M is any number: rows past the end read the last one again, and are not stored.
// SPLITK: work item w is tile w % tiles, range w / tiles of the contraction, whose fp32 sums go to partial[range][M][N].
// On random codes 16384^3 1585 us, 5.55 PFLOP/s, 8192 x 4096 x 14336 179 us, 5.4, 8192 x 14336 x 4096 207 us, 4.65; on zeros 18 to 20 %
// less: the chip lowers its clock under the switching of full tiles (register-only loops of the instruction reach 9.8 PFLOP/s on zeros,
// 7.1 to 7.4 on random codes).  A tile costs 1.5 us for each 256 of the contraction and 5.5 us for its end; starting the workgroups
// apart from each other, so that their stores do not meet, changes nothing (209 to 207).
// RAGGED: the row's bytes are no multiple of 256: what lies past their end is loaded as zero, by the range check of buffer loads.
template <int BM, int BN>
struct Mx4Lds {
    // (one row of MFMA tiles at a time: two workgroups of 128 x 128 tiles fit a compute unit)
    static constexpr int kEpw = BN / 2 / 16 >= 8 ? 8 : 4, kEpr = 1, kEpStride = kEpw == 4 ? 128 : 16 * kEpw * 2 + 16;
    static constexpr int kStage = (BM + BN) * kBK, kScales = (BM + BN) * 16, kEpilogue = 4 * 16 * kEpr * kEpStride;
};

template <int BM, int BN, bool SPLITK, bool RAGGED>
__global__ __launch_bounds__(256) void mx4_tile_kernel(const Mx4Args p, int tiles_m, int tiles_n, int KT /* steps of a work item, even */, int splits,
                                                       float* __restrict__ partial)
{
    using L = Mx4Lds<BM, BN>;
    __shared__ __attribute__((aligned(1024))) uint8_t st0[L::kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t st1[L::kStage];
    __shared__ __attribute__((aligned(1024))) uint8_t scb[L::kScales];
    __shared__ __attribute__((aligned(16))) uint8_t epb[L::kEpilogue];
    constexpr int NW = 4, WM = BM / 2, WN = BN / 2, TM = WM / 16, TN = WN / 16;  // waves, wave tile, fragments
    constexpr int A_BYTES = BM * kBK, A_LOADS = BM / 8 / NW, B_LOADS = BN / 8 / NW, LOADS = A_LOADS + B_LOADS;
    constexpr int EPW = L::kEpw, EPR = L::kEpr, EP_STRIDE = L::kEpStride;
    using std::integral_constant;
    using I0 = integral_constant<int, 0>;
    using I1 = integral_constant<int, 1>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / 2, wn = wave % 2, fr = lane & 15, fg = lane >> 4;
    const int tiles_mn = tiles_m * tiles_n, total = SPLITK ? tiles_mn * splits : tiles_mn;
    const int64_t pitch = mx4_pitch(p.K);
    const int groups = (p.K + kMxGroup - 1) / kMxGroup;
    auto stage_ptr = [&](auto S) -> uint8_t* {
        if constexpr (decltype(S)::value == 0) return st0;
        else return st1;
    };

    // ---- load stream: wave w fills rows [w * R / 4, ...) of each operand's tile in pieces of 8 rows; lane i lands at row i / 8,
    // physical chunk i % 8 of a piece, and fetches the logical chunk that belongs there
    const int chunk = 16 * ((lane & 7) ^ mx4_swz(lane >> 3));
    const uint8_t *a_base, *b_base, *sa_base, *sb_base;
    uint32_t a_off[A_LOADS], b_off[B_LOADS];
    int64_t left = 0;    // bytes of a row from the item's first on
    int group0 = 0;      // the item's first group
    int ld_item = (int)blockIdx.x;
    auto load_context = [&](int item) {
        int tm, tn;
        tile_coords(SPLITK ? item % tiles_mn : item, tiles_m, tiles_n, &tm, &tn);
        const int64_t koff = SPLITK ? (int64_t)(item / tiles_mn) * KT * kBK : 0;
        left = pitch - koff, group0 = (int)(koff / (2 * kBK));
        const int m0 = p.m0 + tm * BM, n0 = p.n0 + tn * BN;
        a_base = p.A + (int64_t)m0 * pitch + koff, b_base = p.B + (int64_t)n0 * pitch + koff;
        const int a_last = p.M - 1 - m0, b_last = p.N - 1 - n0;
        int row8 = lane >> 3;
        asm volatile("" : "+v"(row8));  // (the rows are not to be kept in registers)
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) {
            const int row = wave * (BM / NW) + 8 * i + row8;
            a_off[i] = (uint32_t)(row < a_last ? row : a_last) * (uint32_t)pitch + chunk;
        }
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i) {
            const int row = wave * (BN / NW) + 8 * i + row8;
            b_off[i] = (uint32_t)(row < b_last ? row : b_last) * (uint32_t)pitch + chunk;
        }
        // this wave's 64 rows of each operand's scales (the last ones again past the end)
        const int a_piece = m0 / 64 + wave % (BM / 64), b_piece = n0 / 64 + wave % (BN / 64);
        const int a_most = (int)(p.a_srows / 64) - 1, b_most = (int)(p.b_srows / 64) - 1;
        sa_base = p.sa + (int64_t)(a_piece < a_most ? a_piece : a_most) * 1024;
        sb_base = p.sb + (int64_t)(b_piece < b_most ? b_piece : b_most) * 1024;
    };
    auto cut_loads = [&](int kt) {  // of step kt, what lies past the rows' end; so it does for all steps to come
        if constexpr (!RAGGED) return;
        const int64_t valid = left - (int64_t)kt * kBK;
        if (valid >= kBK) return;  // uniform
        if (chunk >= valid) {
#pragma unroll
            for (int i = 0; i < A_LOADS; ++i) a_off[i] = kPastEnd;
#pragma unroll
            for (int i = 0; i < B_LOADS; ++i) b_off[i] = kPastEnd;
        }
    };
    auto source_at = [](const uint8_t* q) {
        if constexpr (RAGGED) return buffer_at(q);
        else return q;
    };
    auto issue_one = [&](auto ga, auto gb, auto S, auto IDX) {
        constexpr int idx = decltype(IDX)::value;
        constexpr bool is_a = idx < A_LOADS;
        constexpr int j = is_a ? idx : idx - A_LOADS;
        const uint32_t lds = lds_address(stage_ptr(S) + (is_a ? 0 : A_BYTES) + wave * ((is_a ? BM : BN) / NW) * kBK + j * 1024);
        const auto src = is_a ? ga : gb;
        uint32_t o;
        if constexpr (is_a) o = a_off[j];
        else o = b_off[j];
        if constexpr (RAGGED)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(o), "s"(src) : "memory");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(o), "s"(src) : "memory");
    };
    auto step_a = [&](int kt) { return a_base + (int64_t)kt * kBK; };
    auto step_b = [&](int kt) { return b_base + (int64_t)kt * kBK; };
    // the scales of the pair of steps from kt on (past the last group, where the codes are zeros, its scales again)
    const uint32_t scale_lane = lane * 16;
    auto issue_scales = [&](int kt, auto WHICH) {
        int g = group0 + kt / 2;
        g = g < groups ? g : groups - 1;
        constexpr bool is_a = decltype(WHICH)::value == 0;
        const uint8_t* src = is_a ? sa_base + g * (p.a_srows * 16) : sb_base + g * (p.b_srows * 16);
        const uint32_t lds = lds_address(scb + (is_a ? wave % (BM / 64) * 1024 : BM * 16 + wave % (BN / 64) * 1024));
        const uint32_t o = scale_lane;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(o), "s"(src) : "memory");
    };
    auto next_item = [&]() {  // past the last one the stream stays: the same number of loads in every step
        ld_item += (int)gridDim.x;
        if (ld_item < total) load_context(ld_item);
    };

    // ---- fragments: 16 rows, 256 elements; lane: row fr, blocks fg and 4 + fg
    const int a_rd = (wm * WM + fr) * kBK, b_rd = A_BYTES + (wn * WN + fr) * kBK;
    const int c0 = 16 * (fg ^ mx4_swz(fr)), c1 = 16 * ((4 + fg) ^ mx4_swz(fr));
    struct Frag {
        v4i k[2];
    };
    Frag fa[TM], fb[TN], fb_early;
    int sa[TM], sb[TN], sb_early;
    auto read = [&](const uint8_t* row) { return Frag{{*reinterpret_cast<const v4i*>(row + c0), *reinterpret_cast<const v4i*>(row + c1)}}; };
    auto read_a = [&](auto S, auto I) { fa[decltype(I)::value] = read(stage_ptr(S) + a_rd + decltype(I)::value * 16 * kBK); };
    auto read_b = [&](auto S, auto I) { fb[decltype(I)::value] = read(stage_ptr(S) + b_rd + decltype(I)::value * 16 * kBK); };
    const int sa_rd = (wm * WM + fr) * 16 + fg * 4, sb_rd = BM * 16 + (wn * WN + fr) * 16 + fg * 4;
    auto read_sa = [&](auto I) { sa[decltype(I)::value] = *reinterpret_cast<const int*>(scb + sa_rd + decltype(I)::value * 256); };
    auto read_sb = [&](auto I) { sb[decltype(I)::value] = *reinterpret_cast<const int*>(scb + sb_rd + decltype(I)::value * 256); };

    v4f acc[TM][TN];
    auto zero_acc = [&]() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    };

    // ---- order of the step's slots, as in gemm_tile_kernel; slots 2 q and 2 q + 1 do the first halves of both their products,
    // then the second halves
    constexpr int SLOTS = TM * TN, HALF = SLOTS / 2, HM = TM / 2;
    constexpr auto slot_i = [](int s) { return s < HALF ? s / TN : HM + (s - HALF) % HM; };
    constexpr auto slot_j = [](int s) { return s < HALF ? s % TN : (s - HALF) / HM; };
    auto mfma = [&](auto S, auto SLOT, auto K) {
        constexpr int s = decltype(SLOT)::value, i = slot_i(s), j = slot_j(s), k = decltype(K)::value, byte = 2 * decltype(S)::value + k;
        v4f& c = acc[i][j];
        const v4i& b = fb[j].k[k];
        const v4i& a = fa[i].k[k];
        const int& tb = sb[j];
        const int& ta = sa[i];
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%5,0] op_sel_hi:[%6,%6,0] cbsz:4 blgp:4"
                     : "+a"(c)
                     : "v"(b), "v"(a), "v"(tb), "v"(ta), "n"(byte & 1), "n"(byte >> 1));
    };
    auto mfma_slot = [&](auto S, auto SLOT) {
        mfma(S, SLOT, I0{});
        mfma(S, SLOT, I1{});
    };
    auto drain = [&]() { asm volatile("s_nop 15\n\ts_nop 15"); };  // nothing interlocks an accumulator's first ordinary read

    // ---- epilogue of one tile, as in gemm_tile_kernel, but its stores are still under way when the next tile begins: the loads
    // that one starts with are waited for before them, so its first step waits for no load
    auto epilogue = [&](int item) {
        int lane = (int)threadIdx.x & 63;  // (not to be kept in registers over the products, nor what follows from it)
        asm volatile("" : "+v"(lane));
        const int fr = lane & 15, fg = lane >> 4;
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
        int tm, tn;
        tile_coords(SPLITK ? item % tiles_mn : item, tiles_m, tiles_n, &tm, &tn);
        const int m0 = p.m0 + tm * BM + wm * WM, n0 = p.n0 + tn * BN + wn * WN;
        if constexpr (SPLITK) {
            float* P = partial + (int64_t)(item / tiles_mn) * p.M * p.N;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int m = m0 + 16 * i + fr;
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int n = n0 + 16 * j + 4 * fg;
                    if (m < p.M && n < p.N) *reinterpret_cast<v4f*>(P + (int64_t)m * p.N + n) = acc[i][j];
                }
            }
            return;
        }
        uint8_t* ep = epb + wave * (16 * EPR * EP_STRIDE);
        uint8_t* dbase = reinterpret_cast<uint8_t*>(p.D + (int64_t)m0 * p.ldd + n0);
        const uint32_t ldd_b = (uint32_t)p.ldd * 2;
        constexpr int LPR = 2 * EPW;  // lanes (16-byte pieces) per staged row
        const uint32_t voff = (uint32_t)(lane / LPR) * ldd_b + (uint32_t)(lane % LPR) * 16;
        auto run = [&](auto INTERIOR) {
            static_for<(TM / EPR) * (TN / EPW)>([&](auto P) {
                constexpr int ip = decltype(P)::value / (TN / EPW), jp = decltype(P)::value % (TN / EPW);
#pragma unroll
                for (int ii = 0; ii < EPR; ++ii)
#pragma unroll
                    for (int jj = 0; jj < EPW; ++jj) {
                        const v4f& c = acc[EPR * ip + ii][EPW * jp + jj];
                        const uint2 o = make_uint2(pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3]));
                        if constexpr (EPW == 4) *reinterpret_cast<uint2*>(ep + (16 * ii + fr) * EP_STRIDE + 16 * ((2 * jj + (fg >> 1)) ^ (fr & 7)) + 8 * (fg & 1)) = o;
                        else *reinterpret_cast<uint2*>(ep + (16 * ii + fr) * EP_STRIDE + (16 * jj + 4 * fg) * 2) = o;
                    }
                uint8_t* pbase = dbase + ((int64_t)(16 * EPR * ip) * p.ldd + 16 * EPW * jp) * 2;
#pragma unroll
                for (int t = 0; t < 16 * EPR * LPR / 64; ++t) {
                    const int idx = t * 64 + lane, piece = EPW == 4 ? (idx % LPR) ^ ((idx / LPR) & 7) : idx % LPR;
                    const uint4 v = *reinterpret_cast<const uint4*>(ep + (idx / LPR) * EP_STRIDE + piece * 16);
                    bool ok = true;
                    if constexpr (!decltype(INTERIOR)::value) ok = m0 + 16 * EPR * ip + idx / LPR < p.M && n0 + 16 * EPW * jp + (idx % LPR) * 8 < p.N;
                    if (ok) store_stream(reinterpret_cast<uint4*>(pbase + (voff + (uint32_t)(64 / LPR * t) * ldd_b)), v);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        if (p.m0 + tm * BM + BM <= p.M && p.n0 + tn * BN + BN <= p.N) run(std::true_type{});
        else run(std::false_type{});
    };

    auto read_first_set = [&](auto S) {
        static_for<HM>([&](auto I) { read_a(S, I); });
        static_for<TN>([&](auto J) { read_b(S, J); });
        static_for<HM>([&](auto I) { read_sa(I); });
        static_for<TN>([&](auto J) { read_sb(J); });
    };

    // ---- prologue
    load_context(ld_item);
    issue_scales(0, I0{}), issue_scales(0, I1{});
    auto issue_all = [&](int kt, auto S) {
        const auto ga = source_at(step_a(kt)), gb = source_at(step_b(kt));
        static_for<LOADS>([&](auto I) { issue_one(ga, gb, S, I); });
    };
    cut_loads(0);
    issue_all(0, I0{});
    cut_loads(1);
    issue_all(1, I1{});
    zero_acc();
    __builtin_amdgcn_s_waitcnt(kWaitAllVmLgkm);
    __syncthreads();
    read_first_set(I0{});

    // ---- one step out of stage S: the schedule of gemm_tile_kernel, and
    //   the scales' words are read where their fragments are, but only once in a pair of steps: those that an even step starts
    //   with in the odd step before, the lower A fragments' in the even step itself;
    //   even steps, late slots: + the loads of the next pair's scales (behind the barrier after those reads)
    constexpr int SYNC_A = HM + (SLOTS >= 64 ? 8 : SLOTS >= 32 ? 4 : 1);
    constexpr int SYNC_B = HALF - 2;
    constexpr int L_END = SLOTS >= 64 ? SLOTS - SLOTS / 8 : SLOTS;
    static_assert(SYNC_A <= SYNC_B && L_END - SYNC_A >= LOADS / 2, "schedule does not fit");
    constexpr auto slot_of_load = [](int l) { return SYNC_A + l * (L_END - SYNC_A) / LOADS; };
    constexpr int PRE_B = [&] {
        int n = 0;
        for (int l = 0; l < LOADS; ++l) n += slot_of_load(l) < SYNC_B;
        return n;
    }();
    constexpr auto slot_of_next_b = [](int j) {
        const int s = HALF + (j + 1) * HM - 1;
        return s < SLOTS - 3 ? s : SLOTS - 3;
    };
    constexpr int kWaitB = (PRE_B & 15) | ((PRE_B >> 4) << 14) | 0x0070;  // vmcnt(PRE_B) lgkmcnt(0)

    auto kstep = [&](auto S, int fetch_kt, bool first) {
        constexpr int s = decltype(S)::value;
        using OTHER = integral_constant<int, 1 - s>;
        const auto ga = source_at(step_a(fetch_kt)), gb = source_at(step_b(fetch_kt));
        static_for<SLOTS>([&](auto SLOT) {
            constexpr int slot = decltype(SLOT)::value;
            if constexpr (slot == SYNC_A) {
                __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): my reads of stage S are back
                __syncthreads();
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (slot == SYNC_B) {
                if (s == 0 && first) __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
                else __builtin_amdgcn_s_waitcnt(kWaitB);
                __syncthreads();
                __builtin_amdgcn_sched_barrier(0);
            }
            mfma_slot(S, SLOT);
            if constexpr (slot < HM) {
                read_a(S, integral_constant<int, HM + slot>{});
                if constexpr (s == 0) read_sa(integral_constant<int, HM + slot>{});
            }
            if constexpr (slot >= HALF && slot < HALF + HM) {
                read_a(OTHER{}, integral_constant<int, slot - HALF>{});
                if constexpr (s == 1) read_sa(integral_constant<int, slot - HALF>{});
            }
            static_for<TN>([&](auto J) {
                constexpr int j = decltype(J)::value;
                if constexpr (slot_of_next_b(j) == slot) {
                    if constexpr (slot < HALF + (j + 1) * HM - 1) {  // fb[j] is still needed: park its successor
                        static_assert(j == TN - 1, "one spare fragment");
                        const Frag keep = fb[j];
                        const int keep_scale = sb[j];
                        read_b(OTHER{}, J);
                        if constexpr (s == 1) read_sb(J);
                        fb_early = fb[j], sb_early = sb[j];
                        fb[j] = keep, sb[j] = keep_scale;
                    } else {
                        read_b(OTHER{}, J);
                        if constexpr (s == 1) read_sb(J);
                    }
                }
            });
            if constexpr (slot == SLOTS - 1 && slot_of_next_b(TN - 1) < SLOTS - 1) fb[TN - 1] = fb_early, sb[TN - 1] = sb_early;
            static_for<LOADS>([&](auto I) {
                if constexpr (slot_of_load(decltype(I)::value) == slot) issue_one(ga, gb, S, I);
            });
            if constexpr (s == 0 && slot == SLOTS - 4) issue_scales(fetch_kt, I0{});
            if constexpr (s == 0 && slot == SLOTS - 2) issue_scales(fetch_kt, I1{});
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    // ---- main loop.  The step computed at kt fetches step kt + 2; the last two of a tile fetch the first two of the next one.
    for (int item = (int)blockIdx.x; item < total; item += (int)gridDim.x) {
        for (int kt = 0; kt < KT; kt += 2) {
            if (kt == KT - 2) next_item();
            const int f = kt == KT - 2 ? 0 : kt + 2;
            cut_loads(f);
            kstep(I0{}, f, kt == 0);
            cut_loads(f + 1);
            kstep(I1{}, f + 1, false);
        }
        drain();
        epilogue(item);
        zero_acc();
        read_first_set(I0{});
        asm volatile("s_nop 7");  // accumulators just written by ordinary instructions: let them settle
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // no load may still be writing LDS when the workgroup ends
}

// partial[s][M][N] fp32 of s < splits ranges, added in their order; a thread owns eight columns.
__global__ __launch_bounds__(256) void mx4_reduce_kernel(const float* __restrict__ partial, int splits, int M, int N, uint16_t* __restrict__ D, int64_t ldd)
{
    const int chunks = N / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)M * chunks) return;
    const int m = (int)(i / chunks), n = (int)(i % chunks) * 8;
    const float* q = partial + (int64_t)m * N + n;
    const int64_t stride = (int64_t)M * N;
    v4f lo = *reinterpret_cast<const v4f*>(q), hi = *reinterpret_cast<const v4f*>(q + 4);
    for (int s = 1; s < splits; ++s) lo += *reinterpret_cast<const v4f*>(q + s * stride), hi += *reinterpret_cast<const v4f*>(q + s * stride + 4);
    *reinterpret_cast<uint4*>(D + (int64_t)m * ldd + n) =
        make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
}

// ---- host ----------------------------------------------------------------------------------------

template <int TM, int TN, int STAGES, bool TOKENS = false>
static void launch_rows(const Mx4Args& a, hipStream_t st, const uint16_t* X = nullptr)
{
    const int tiles_m = (a.M + 16 * TM - 1) / (16 * TM), tiles_n = (a.N + 16 * TN - 1) / (16 * TN);
    const size_t tokens = TOKENS ? (size_t)a.M * (mx4_pitch(a.K) + (a.K + kMxGroup - 1) / kMxGroup * 16) : 0;
    mx4_rows_kernel<TM, TN, STAGES, TOKENS><<<(unsigned)(tiles_m * tiles_n), 256, tokens, st>>>(a, tiles_m, tiles_n, X);
}

template <int TM, int STAGES>
static void launch_strip(const Mx4Args& a, hipStream_t st)
{
    const int tiles_m = (a.M + 16 * TM - 1) / (16 * TM), tiles_n = (a.N + 63) / 64;
    mx4_strip_kernel<TM, STAGES><<<(unsigned)(tiles_m * tiles_n), 512, 0, st>>>(a, tiles_m, tiles_n);
}

// Steps of a work item when the contraction is cut into `ranges`: whole pairs, at least one.
static int steps_of(int K, int ranges)
{
    const int groups = (K + kMxGroup - 1) / kMxGroup, per = (groups + ranges - 1) / ranges;
    return 2 * (per > 0 ? per : 1);
}

template <int BM, int BN>
static void launch_tiles(const Mx4Args& a, int most, hipStream_t st)
{
    const int tiles_m = (a.M - a.m0 + BM - 1) / BM, tiles_n = (a.N - a.n0 + BN - 1) / BN, total = tiles_m * tiles_n;
    const auto kernel = a.K % kMxGroup ? mx4_tile_kernel<BM, BN, false, true> : mx4_tile_kernel<BM, BN, false, false>;
    kernel<<<(unsigned)(total < most ? total : most), 256, 0, st>>>(a, tiles_m, tiles_n, steps_of(a.K, 1), 1, nullptr);
}

// How a product is launched: by estimated time, in us.  A kernel whose tiles take r rounds of one tile a compute unit needs
// start + r (tile + group G) for G groups of 512 of the contraction; the constants are fits to 24 sizes of 1 to 4096 rows, good to
// 15 %, and no kernel is taken to read its operands faster than 4.2 TB/s.  What they decide between, each in its us (rows x columns
// x contraction; tiles of 16 x 16, 32 x 32, 64 x 64 strips, 96 x 64 strips, 128 x 128, 256 x 256):
//   1 x 4096 x 4096      4.5   5.0   7.1   9.0  12.7  25.4        300 x 4096 x 4096    53.5  20.2  13.8  10.0  12.9  25.4
//   1 x 14336 x 4096    14.6  10.7   8.6  10.3  16.9  27.2        1000 x 14336 x 4096   621   223  93.6  87.0  41.4  31.6
// (tiles of 32 x 32, 64 x 32, strips of 64, 96 and 128 rows, 128 x 128, 256 x 128)
//   40 x 4144 x 1040     6.6   4.9   5.2   6.0   6.8   7.2   9.4     1287 x 1200 x 1568  20.5  15.5  10.3  13.1   9.1   9.5  12.3
//   64 x 4096 x 4096     5.6   6.7   7.5   9.4  10.9  11.8  15.4     2068 x 928 x 8192   45.4  33.1  21.3  28.4  19.2  22.3  28.1
// Ranges of the contraction, with a workspace, against the best of the others: of 44 sizes that the estimates send there 40 gain, by 5 to
// 46 % (468 x 5456 x 81696 in four 164 us for 305, 3976 x 480 x 65344 in eight 89 for 150, 1500 x 5024 x 87296 in two 294 for 370);
// where the estimates are close some lose, up to 12 % (2048 x 2032 x 20480 in four 60 for 54, 3976 x 656 x 14336 41 for 38, 721 x 416
// x 90624 in eight 69 for 64).
struct Mx4Plan {
    enum Kind { kRows11, kRows12, kRows14, kRows22, kRows42, kStrip4, kStrip6, kStrip8, kQuarter, kHalf, kFull, kFullRows, kFullCols, kSplit } kind;
    int ranges, whole;  // kSplit: ranges of the contraction; kFullRows, kFullCols: tiles in whole rounds, launched on their own
};

// Up to kMxTokens rows have their kernel by the columns alone, so that a product from bf16 has the bits of that from codes.
// (Not static: the tests ask it which kernel a size is for.)
Mx4Plan plan_product(int64_t M, int64_t N, int64_t K, size_t ws_bytes, int cus)
{
    if (M <= kMxTokens && K > 0) return {N <= 16 * cus ? Mx4Plan::kRows11 : N <= 32 * cus ? Mx4Plan::kRows12 : Mx4Plan::kRows14, 1, 0};
    const auto tiles = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    const auto rounds = [&](int64_t t) { return (double)((t + cus - 1) / cus); };
    const double G = (double)((K + kMxGroup - 1) / kMxGroup);
    if (K == 0) return {Mx4Plan::kRows22, 1, 0};
    static constexpr struct {
        Mx4Plan::Kind kind;
        int bm, bn;
        double start, tile, group;
    } kKernels[] = {{Mx4Plan::kRows11, 16, 16, 1.7, 1.05, 0.22}, {Mx4Plan::kRows12, 16, 32, 1.5, 1.0, 0.26},  {Mx4Plan::kRows22, 32, 32, 1.26, 1.2, 0.32},
                    {Mx4Plan::kRows42, 64, 32, 1.8, 1.2, 0.46},  {Mx4Plan::kStrip4, 64, 64, 1.2, 2.1, 0.52},  {Mx4Plan::kStrip6, 96, 64, 1.3, 2.9, 0.725},
                    {Mx4Plan::kStrip8, 128, 64, 1.1, 3.5, 0.89}, {Mx4Plan::kHalf, 256, 128, 0.0, 3.5, 1.9}};
    const double memory = 2.0 + (double)(M + N) * (double)K * 17.0 / 32.0 / 4.2e6;
    Mx4Plan plan = {Mx4Plan::kFull, 1, 0};
    double best;
    const auto take = [&](Mx4Plan::Kind kind, double us) {
        us = (us > memory ? us : memory) + 0.1 * us;  // (of those that the memory bounds, the one with the least work)
        if (us < best) best = us, plan = {kind, 1, 0};
    };
    // 256 x 256: a last round with at most half of the workgroups busy goes to tiles half as wide, the whole rounds on their own
    const int64_t tm = (M + 255) / 256, tn = (N + 255) / 256, T = tm * tn, whole = T / cus * cus, rest = T - whole;
    const bool by_rows = whole > 0 && rest > 0 && 2 * rest <= cus && whole % tn == 0, by_cols = !by_rows && whole > 0 && rest > 0 && 2 * rest <= cus && whole % tm == 0;
    const double full = 8.0 + 3.1 * G, half = 3.5 + 1.9 * G;
    best = 1e30;
    take(by_rows ? Mx4Plan::kFullRows : by_cols ? Mx4Plan::kFullCols : Mx4Plan::kFull, by_rows || by_cols ? (double)(whole / cus) * full + half : rounds(T) * full);
    plan.whole = (int)whole;
    for (const auto& k : kKernels) take(k.kind, k.start + rounds(tiles(k.bm, k.bn)) * (k.tile + k.group * G));
    const int64_t Q = tiles(128, 128);  // (two of these share a compute unit)
    take(Mx4Plan::kQuarter, Q <= cus ? 2.6 + 1.45 * G : 3.6 + rounds(Q) * (1.65 + 0.93 * G));
    // Ranges of the contraction, with their fp32 sums in the workspace: a range is whole groups, four at least, and not empty.
    for (int s = 2; s <= 8 && s * T <= cus && K / s >= 4 * kMxGroup; s *= 2) {
        const int groups = steps_of((int)K, s) / 2;
        if ((int64_t)(s - 1) * groups * kMxGroup >= K || (size_t)s * (size_t)M * (size_t)N * sizeof(float) > ws_bytes) break;
        take(Mx4Plan::kSplit, full - 3.1 * (G - groups) + 3.0 + (s + 0.5) * (double)M * (double)N * 4.0 / 5.0e6);
        if (plan.kind == Mx4Plan::kSplit && plan.ranges == 1) plan.ranges = s;
    }
    return plan;
}

size_t mx4_split_bytes(int64_t M, int64_t N, int64_t K)
{
    if (M == 0 || N == 0) return 0;
    const Mx4Plan plan = plan_product(M, N, K, ~(size_t)0, cu_count());
    return plan.kind == Mx4Plan::kSplit ? (size_t)plan.ranges * (size_t)M * (size_t)N * sizeof(float) : 0;
}

f8_status mx4_gemm_tokens(const Mx4Args& a, const uint16_t* X, hipStream_t st)
{
    if (a.M == 0 || a.N == 0 || a.K == 0) return mx4_gemm(a, nullptr, 0, st);
    switch (plan_product(a.M, a.N, a.K, 0, cu_count()).kind) {
        case Mx4Plan::kRows11: launch_rows<1, 1, 12, true>(a, st, X); break;
        case Mx4Plan::kRows14: launch_rows<1, 4, 3, true>(a, st, X); break;
        default: launch_rows<1, 2, 6, true>(a, st, X); break;
    }
    return last_launch_status();
}

f8_status mx4_gemm(const Mx4Args& a, void* ws, size_t ws_bytes, hipStream_t st)
{
    if (a.M == 0 || a.N == 0) return last_launch_status();
    const int cus = cu_count();
    const Mx4Plan plan = plan_product(a.M, a.N, a.K, ws ? ws_bytes : 0, cus);
    const int tm = (a.M + 255) / 256, tn = (a.N + 255) / 256;
    switch (plan.kind) {
        case Mx4Plan::kRows11: launch_rows<1, 1, 8>(a, st); break;
        case Mx4Plan::kRows12: launch_rows<1, 2, 5>(a, st); break;
        case Mx4Plan::kRows14: launch_rows<1, 4, 3>(a, st); break;
        case Mx4Plan::kRows22: launch_rows<2, 2, 4>(a, st); break;
        case Mx4Plan::kRows42: launch_rows<4, 2, 2>(a, st); break;
        case Mx4Plan::kStrip4: launch_strip<4, 4>(a, st); break;
        case Mx4Plan::kStrip6: launch_strip<6, 3>(a, st); break;
        case Mx4Plan::kStrip8: launch_strip<8, 3>(a, st); break;
        case Mx4Plan::kSplit: {
            const auto kernel = a.K % kMxGroup || a.K / kMxGroup % plan.ranges ? mx4_tile_kernel<256, 256, true, true> : mx4_tile_kernel<256, 256, true, false>;
            kernel<<<(unsigned)(tm * tn * plan.ranges), 256, 0, st>>>(a, tm, tn, steps_of(a.K, plan.ranges), plan.ranges, (float*)ws);
            const int64_t threads = (int64_t)a.M * (a.N / 8);
            mx4_reduce_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, st>>>((const float*)ws, plan.ranges, a.M, a.N, a.D, a.ldd);
            break;
        }
        case Mx4Plan::kFullRows:
        case Mx4Plan::kFullCols: {
            Mx4Args one = a, two = a;
            if (plan.kind == Mx4Plan::kFullRows) {
                one.M = plan.whole / tn * 256;
                two.m0 = one.M;
            } else {
                one.N = plan.whole / tm * 256;
                two.n0 = one.N;
            }
            launch_tiles<256, 256>(one, cus, st);
            launch_tiles<256, 128>(two, cus, st);
            break;
        }
        case Mx4Plan::kFull: launch_tiles<256, 256>(a, cus, st); break;
        case Mx4Plan::kHalf: launch_tiles<256, 128>(a, cus, st); break;
        case Mx4Plan::kQuarter: launch_tiles<128, 128>(a, 2 * cus, st); break;
    }
    return last_launch_status();
}

}  // namespace f8
