// Quantisation to microscaled 4-bit blocks and back, and the linear on them:
//   a block's scale is 2^e with e = floor(log2(largest magnitude)) - 2 (at least -127), so that the largest lies in [4, 8);
//   code = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| 2^-e, ties to the even code, above 6: 6; a block with an infinity or
//   a NaN has the scale NaN.
// Forward Y = X4 W4^T with blocks along K; backward dX = dY4 W4^T with blocks along N and dW = dY4^T X4 with blocks along M: a
// tensor's other orientation has codes of its own, and one reading of the tensor gives both.
// The cast is bound by memory: 2 bytes an element read, 17/32 for each orientation written.  8192 x 14336, us: along the rows 46.5 (6.4
// TB/s), across them 65 (4.6), both 82 (4.4: half lines of both orientations' codes, and bytes of scales); back to bf16 102 (2.9).
#include "f8_device.hpp"
#include "f8_mx4.hpp"
#include "f8_mx4_device.hpp"

namespace f8 {

struct Mx4Cast {
    const uint16_t* x;
    int64_t ld;
    int rows, cols;
    uint8_t *q, *s, *q_t, *s_t;  // either orientation nullable
    int squares, squares_c, blocks;  // squares of 4 x 4 tiles, those side by side
    bool once;                       // loads past the caches
};
// More elements than these are loaded past the caches: 8192 x 14336 along the rows 46.5 us for 55, both ways 84.8 for 86.8, 14336 x
// 4096 both ways 42.1 for 45.3; but 8192 x 4096 along the rows 16.1 for 15.1, across them 22.3 for 18.6.
constexpr int64_t kMxOnce = (int64_t)1 << 25;
template <bool ONCE>
__device__ inline uint4 load_eight(const uint16_t* x)
{
    return ONCE ? load_once(reinterpret_cast<const uint4*>(x)) : *reinterpret_cast<const uint4*>(x);
}

// Tiles of 128 x 128.  Along the rows four threads have a block of 32; for the other orientation the tile goes through LDS, where a
// thread takes 32 rows of two columns.
// A tile writes half lines of codes and a quarter of each 16 bytes of scales: the tiles of a square of 512 x 512 follow each other
// on one XCD (workgroups go round the eight of them), whose L2 joins their pieces.
constexpr int kMxTile = 128;

__device__ inline void mx4_cast_tile(const Mx4Cast& p, int block, uint32_t (&tile)[kMxTile][kMxTile / 2])
{
    const int square = block / 128 * 8 + block % 8, in = block / 8 % 16;
    if (square >= p.squares) return;
    const int t = threadIdx.x, r0 = (square / p.squares_c * 4 + in / 4) * kMxTile, c0 = (square % p.squares_c * 4 + in % 4) * kMxTile;
    if ((r0 >= p.rows && !(p.q_t && c0 < mx4_rows(p.cols))) || (c0 >= p.cols && !(p.q && r0 < mx4_rows(p.rows)))) return;  // not even padding
    const bool turn = p.q_t != nullptr;
    const int64_t pitch = mx4_pitch(p.cols), srows = mx4_rows(p.rows);
    // 16 threads take a row's 16-byte chunks, four of them a block
    constexpr int PER = kMxTile * kMxTile / 8 / 256;
    const int k = t % 16, col = c0 + 8 * k;
    uint4 v[PER];
    const auto load = [&](auto ONCE) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int row = r0 + 16 * i + t / 16;
            v[i] = make_uint4(0, 0, 0, 0);
            if (row < p.rows && col < p.cols) v[i] = load_eight<ONCE()>(p.x + (int64_t)row * p.ld + col);
        }
    };
    if (p.once) load(std::true_type{});
    else load(std::false_type{});
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = 16 * i + t / 16, row = r0 + r;
        if (turn) *reinterpret_cast<uint4*>(&tile[r][4 * k]) = v[i];
        if (p.q) {
            const uint32_t code = mx4_scale_of_quad(v[i]);
            const bool real = row < p.rows && col / kMxBlock * kMxBlock < p.cols;
            if (real) *reinterpret_cast<uint32_t*>(p.q + row * pitch + col / 2) = mx4_encode8(v[i], code);
            // (rows of padding too, and blocks up to the group's end)
            if (k % 4 == 0 && row < srows && col < (p.cols + kMxGroup - 1) / kMxGroup * kMxGroup)
                p.s[mx4_scale_at(srows, row, col / kMxBlock)] = (uint8_t)(real ? code : 127);
        }
    }
    if (!turn) return;
    __syncthreads();
    const int wave = t / kWave, lane = t % kWave, rb = r0 / kMxBlock + wave;  // 32 rows of the columns 2 lane, 2 lane + 1
    const int64_t pitch_t = mx4_pitch(p.rows), srows_t = mx4_rows(p.cols);
    uint32_t w[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) w[k] = tile[32 * wave + k][lane];
    uint4 turned[2][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = w[8 * k + 2 * j], b = w[8 * k + 2 * j + 1];
            lo[j] = __builtin_amdgcn_perm(b, a, 0x05040100), hi[j] = __builtin_amdgcn_perm(b, a, 0x07060302);  // the halves of both
        }
        turned[0][k] = make_uint4(lo[0], lo[1], lo[2], lo[3]), turned[1][k] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    }
    // The four waves' codes of a column lie side by side: they meet in LDS, each wave's in the place of the rows that it alone has
    // read, and four lanes write 64 bytes (16 bytes a lane, each to another line: 8192 x 14336 both ways 87.6 us for 82.2, across
    // alone 72.8 for 65.1).
    // Column c's piece at 16-byte word (c + 2 wave) % 128, so that a quad's four pieces and the next one's are in different banks.
    uint4* const codes = reinterpret_cast<uint4*>(&tile[32 * wave][0]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int col = c0 + 2 * lane + h;
        const bool real = col < p.cols && rb * kMxBlock < p.rows;
        const uint32_t code = mx4_scale_of(turned[h]);
        codes[(2 * lane + h + 2 * wave) % kMxTile] = mx4_encode(turned[h], code);
        if (col < srows_t && rb * kMxBlock < (p.rows + kMxGroup - 1) / kMxGroup * kMxGroup) p.s_t[mx4_scale_at(srows_t, col, rb)] = (uint8_t)(real ? code : 127);
    }
    __syncthreads();
    const int piece = t % 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = t / 4 + 64 * i;
        const uint4 o = reinterpret_cast<const uint4*>(&tile[32 * piece][0])[(c + 2 * piece) % kMxTile];
        if (c0 + c < p.cols && r0 + 32 * piece < p.rows) *reinterpret_cast<uint4*>(p.q_t + (c0 + c) * pitch_t + (int64_t)(r0 / kMxBlock + piece) * 16) = o;
    }
}

// One or two tensors: the first a.blocks blocks of the grid are the first one's.
__global__ __launch_bounds__(256) void mx4_cast_kernel(const Mx4Cast a, const Mx4Cast b)
{
    __shared__ __attribute__((aligned(16))) uint32_t tile[kMxTile][kMxTile / 2];
    if ((int)blockIdx.x < a.blocks) mx4_cast_tile(a, (int)blockIdx.x, tile);
    else mx4_cast_tile(b, (int)blockIdx.x - a.blocks, tile);
}

// One orientation alone, along the rows: a wave has a group of 512 elements of ROWS rows, and writes whole pieces of codes and scales.
template <int ROWS>
__global__ __launch_bounds__(256) void mx4_cast_rows_kernel(const Mx4Cast p, int groups)
{
    const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, srows = mx4_rows(p.rows);
    const int64_t row0 = w / groups * ROWS;
    if (row0 >= srows) return;
    const int g = (int)(w % groups), lane = threadIdx.x % kWave, col = g * kMxGroup + 8 * lane, b = lane / 4;
    const int64_t pitch = mx4_pitch(p.cols);
    uint4 v[ROWS];
    const auto load = [&](auto ONCE) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (row0 + i < p.rows && col < p.cols) v[i] = load_eight<ONCE()>(p.x + (row0 + i) * p.ld + col);
        }
    };
    if (ROWS > 1 && p.once) load(std::true_type{});
    else load(std::false_type{});
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const uint32_t code = mx4_scale_of_quad(v[i]);
        const bool real = row0 + i < p.rows && col / kMxBlock * kMxBlock < p.cols;
        if (real) *reinterpret_cast<uint32_t*>(p.q + (row0 + i) * pitch + col / 2) = mx4_encode8(v[i], code);
        if (lane % 4 == 0) p.s[((int64_t)g * srows + row0 + i) * 16 + 4 * (b % 4) + b / 4] = (uint8_t)(real ? code : 127);
    }
}

__global__ __launch_bounds__(256) void mx4_decode_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int rows, int cols, uint16_t* out, int64_t ldo)
{
    const int blocks = (cols + kMxBlock - 1) / kMxBlock;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)rows * blocks) return;
    const int row = (int)(i / blocks), b = (int)(i % blocks);
    const uint4 codes = *reinterpret_cast<const uint4*>(q + row * mx4_pitch(cols) + 16 * (int64_t)b);
    const uint32_t e = s[mx4_scale_at(mx4_rows(rows), row, b)];
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (32 * b + 8 * k < cols) *reinterpret_cast<uint4*>(out + (int64_t)row * ldo + 32 * b + 8 * k) = mx4_decode8(w[k], e);
}

// ---- host ----------------------------------------------------------------------------------------

// (Squares of 512 x 512 hold the codes of both orientations, their padding and the scales': whole groups of 512, and 64 rows.)
// No squares, and no launch, if there is nothing to read or nowhere to write to.
static Mx4Cast cast_of(const void* x, int64_t rows, int64_t cols, int64_t ld, const f8_mx4& o)
{
    const int64_t across = (cols + kMxGroup - 1) / kMxGroup, squares = rows > 0 && cols > 0 && (o.q || o.q_t) ? (rows + kMxGroup - 1) / kMxGroup * across : 0;
    return {(const uint16_t*)x, ld, (int)rows, (int)cols, o.q, o.s, o.q_t, o.s_t, (int)squares, (int)across, (int)((squares + 7) / 8 * 128),
            rows * cols > kMxOnce};
}
static bool too_many(int64_t rows, int64_t cols) { return (rows / kMxGroup + 1) * (cols / kMxGroup + 1) > 0x2FFFFFF; }
constexpr int64_t kFewWaves = 16384;
static void launch_cast(const Mx4Cast& a, const Mx4Cast& b, hipStream_t st)
{
    if (a.blocks > 0 && b.blocks == 0 && !a.q_t) {
        // (a row for each wave while there are few)
        const int groups = (a.cols + kMxGroup - 1) / kMxGroup;
        const int64_t all = mx4_rows(a.rows) * groups;
        if (all <= kFewWaves) mx4_cast_rows_kernel<1><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a, groups);
        else mx4_cast_rows_kernel<4><<<(unsigned)((all / 4 + 3) / 4), 256, 0, st>>>(a, groups);
        return;
    }
    if (a.blocks + b.blocks > 0) mx4_cast_kernel<<<(unsigned)(a.blocks + b.blocks), 256, 0, st>>>(a, b);
}

// The pairs that are needed are there (of an empty tensor none is: it has no bytes).
static f8_status check_codes(const f8_mx4* t, int64_t rows, int64_t cols, bool along_cols, bool along_rows)
{
    if (rows == 0 || cols == 0) along_cols = along_rows = false;
    if (!t || (along_cols && (!t->q || !t->s)) || (along_rows && (!t->q_t || !t->s_t))) return F8_ERR_NULL;
    if ((t->q != nullptr) != (t->s != nullptr) || (t->q_t != nullptr) != (t->s_t != nullptr)) return F8_ERR_NULL;
    if (!aligned16(t->q) || !aligned16(t->s) || !aligned16(t->q_t) || !aligned16(t->s_t)) return F8_ERR_ALIGN;
    return F8_OK;
}
static bool bad_desc(const f8_mx4_desc* d)
{
    return d->M < 0 || d->K < 0 || d->N < 0 || d->M >= kMxMax || d->K >= kMxMax || d->N >= kMxMax || (d->K % 16) || (d->N % 16) || too_many(d->M, d->K) ||
           too_many(d->M, d->N) || too_many(d->N, d->K);
}

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_mx4_scale_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows >= kMxMax || cols >= kMxMax) return 0;
    return mx4_scale_bytes(rows, cols);
}

size_t f8_mx4_workspace_bytes(int64_t M, int64_t K, int64_t N)
{
    size_t most = kMinWorkspaceBytes;
    if (M < 0 || K < 0 || N < 0 || M >= kMxMax || K >= kMxMax || N >= kMxMax) return most;
    for (const size_t b : {mx4_split_bytes(M, N, K), mx4_split_bytes(M, K, N), mx4_split_bytes(N, K, M)}) most = b > most ? b : most;
    return most;
}

f8_status f8_mx4_quantise(const void* x_bf16, int64_t rows, int64_t cols, int64_t ld, const f8_mx4* out, void* stream)
{
    if (rows < 0 || cols < 0 || rows >= kMxMax || cols >= kMxMax || (cols % 16) || ld < cols || (ld % 8) || too_many(rows, cols)) return F8_ERR_SHAPE;
    const f8_status s = check_codes(out, rows, cols, false, false);
    if (s != F8_OK) return s;
    if (rows && cols && !out->q && !out->q_t) return F8_ERR_NULL;
    if (rows && cols && !x_bf16) return F8_ERR_NULL;
    if (!aligned16(x_bf16)) return F8_ERR_ALIGN;
    launch_cast(cast_of(x_bf16, rows, cols, ld, *out), Mx4Cast{}, (hipStream_t)stream);
    return last_launch_status();
}

f8_status f8_mx4_dequantise(const uint8_t* q, const uint8_t* s, int64_t rows, int64_t cols, void* out_bf16, int64_t ldo, void* stream)
{
    if (rows < 0 || cols < 0 || rows >= kMxMax || cols >= kMxMax || (cols % 8) || ldo < cols || (ldo % 8)) return F8_ERR_SHAPE;
    const int64_t blocks = (rows * ((cols + kMxBlock - 1) / kMxBlock) + 255) / 256;
    if (blocks > 0x7FFFFFFF) return F8_ERR_SHAPE;
    if (rows && cols && (!q || !s || !out_bf16)) return F8_ERR_NULL;
    if (!aligned16(q) || !aligned16(s) || !aligned16(out_bf16)) return F8_ERR_ALIGN;
    if (blocks) mx4_decode_kernel<<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(q, s, (int)rows, (int)cols, (uint16_t*)out_bf16, ldo);
    return last_launch_status();
}

f8_status f8_mx4_gemm(int64_t M, int64_t N, int64_t K, const uint8_t* A, const uint8_t* sa, const uint8_t* B, const uint8_t* sb, void* D_bf16, int64_t ldd,
                      void* workspace, size_t workspace_bytes_, void* stream)
{
    if (M < 0 || N < 0 || K < 0 || M >= kMxMax || N >= kMxMax || K >= kMxMax || (N % 16) || ldd < N || (ldd % 8) || ldd >= kMxMax) return F8_ERR_SHAPE;
    if (((M + 63) / 64) * ((N + 63) / 64) > (int64_t)0x7FFFFFFF) return F8_ERR_SHAPE;
    if (M && N && (!D_bf16 || (K && (!A || !sa || !B || !sb)))) return F8_ERR_NULL;
    if (!aligned16(A) || !aligned16(sa) || !aligned16(B) || !aligned16(sb) || !aligned16(D_bf16) || !aligned16(workspace)) return F8_ERR_ALIGN;
    return mx4_gemm({(int)M, (int)N, (int)K, A, sa, B, sb, (uint16_t*)D_bf16, ldd}, workspace, workspace ? workspace_bytes_ : 0, (hipStream_t)stream);
}

f8_status f8_mx4_linear_fwd(const f8_mx4_desc* d, const void* X, const void* W, void* Y, const f8_mx4_saved* saved, void* workspace, size_t workspace_bytes_,
                            void* stream)
{
    if (!d || !saved) return F8_ERR_NULL;
    if (bad_desc(d)) return F8_ERR_SHAPE;
    const bool tokens = d->M <= kMxTokens && d->K <= kMxTokenK && !saved->x.q && !saved->x.q_t;  // X's codes are not wanted
    f8_status s = check_codes(&saved->x, d->M, d->K, !tokens, false);
    if (s != F8_OK || (s = check_codes(&saved->w, d->N, d->K, true, false)) != F8_OK) return s;
    if (d->M && ((d->K && !X) || (d->N && !Y))) return F8_ERR_NULL;
    if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || !aligned16(workspace)) return F8_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    const Mx4Cast x = tokens ? Mx4Cast{} : cast_of(X, d->M, d->K, d->K, saved->x), w = W ? cast_of(W, d->N, d->K, d->K, saved->w) : Mx4Cast{};
    launch_cast(x, w, st);
    s = last_launch_status();
    if (s != F8_OK) return s;
    const Mx4Args a = {(int)d->M, (int)d->N, (int)d->K, saved->x.q, saved->x.s, saved->w.q, saved->w.s, (uint16_t*)Y, d->N};
    return tokens ? mx4_gemm_tokens(a, (const uint16_t*)X, st) : mx4_gemm(a, workspace, workspace ? workspace_bytes_ : 0, st);
}

f8_status f8_mx4_linear_bwd(const f8_mx4_desc* d, const void* dY, const f8_mx4_saved* saved, void* dX, void* dW, void* workspace, size_t workspace_bytes_,
                            void* stream)
{
    if (!d || !saved) return F8_ERR_NULL;
    if (bad_desc(d)) return F8_ERR_SHAPE;
    if (!dX && !dW && d->K && (d->M || d->N)) return F8_ERR_NULL;  // (gradients without elements may have no address)
    f8_mx4 dy = saved->dy;
    f8_status s = check_codes(&dy, d->M, d->N, dX != nullptr, dW != nullptr);
    if (s != F8_OK || (dX && (s = check_codes(&saved->w, d->N, d->K, false, true)) != F8_OK) || (dW && (s = check_codes(&saved->x, d->M, d->K, false, true)) != F8_OK)) return s;
    if (d->M && d->N && !dY) return F8_ERR_NULL;
    if (!aligned16(dY) || !aligned16(dX) || !aligned16(dW) || !aligned16(workspace)) return F8_ERR_ALIGN;
    if (!dX) dy.q = dy.s = nullptr;
    if (!dW) dy.q_t = dy.s_t = nullptr;
    hipStream_t st = (hipStream_t)stream;
    const size_t room = workspace ? workspace_bytes_ : 0;
    launch_cast(cast_of(dY, d->M, d->N, d->N, dy), Mx4Cast{}, st);
    s = last_launch_status();
    if (s == F8_OK && dX) s = mx4_gemm({(int)d->M, (int)d->K, (int)d->N, dy.q, dy.s, saved->w.q_t, saved->w.s_t, (uint16_t*)dX, d->K}, workspace, room, st);
    if (s == F8_OK && dW) s = mx4_gemm({(int)d->N, (int)d->K, (int)d->M, dy.q_t, dy.s_t, saved->x.q_t, saved->x.s_t, (uint16_t*)dW, d->K}, workspace, room, st);
    return s;
}

}  // extern "C"
