// Token embeddings and the gradient of their table:
//   out[m] = bf16(scale table[ids[m]]),   dtable[v] = scale (sum of dout[m] over the m with ids[m] = v), zeros where there is none.
// Both are bound by memory: the forward by reading and writing a row for each token, the backward by reading the tokens' rows and
// writing the whole table.  The sums have a fixed order without atomics on results: the tokens are sorted by (id, position), the
// sorted list is cut into pieces of equal length, whatever the ids' frequencies, and a wave adds up a piece's rows for 512
// columns.  An id whose tokens lie in one piece is finished there; the sums of one that goes on over several are left in the
// workspace and joined, in order, by the last launch.
// The sort counts, for each token of a chunk of kChunk, how many of the chunk come before it: two instructions for each pair,
// with the other token's id in a scalar register, in blocks that run beside those that fill the table with zeros.  Longer lists
// are merged by pairs of sorted runs.
// 16384 tokens of 4096 columns, 131072 rows of bf16, us: forward 52 (5.1 TB/s), sort and zeros 151 (7.1 TB/s), two merges 12, pieces 44
// (their rows read once and written once: 5 TB/s), join 9.5.  With a small table the launches have nothing to hide behind: 16384 tokens of
// 1024 columns into 4000 rows 63 us in all, into 32000 rows 72.
#include "f8_rows.hpp"

namespace f8 {

constexpr uint32_t kNoToken = 0xFFFFFFFFu;  // sorts behind every id
constexpr int kChunk = 4096;                // tokens that are sorted by counting (longer chunks cost more than a merge)
constexpr int kSortBlock = 64;              // tokens that a block of the sort places: one a lane, its waves share the others
constexpr int kSortWaves = 4;
constexpr int64_t kEmbedMaxTokens = 1 << 28, kMaxFillBlocks = 1 << 23;

// ---- forward -----------------------------------------------------------------------------------

struct EmbedArgs {
    const int64_t* ids;
    const uint16_t* table;
    int64_t ldt, M, V;
    int dc, strips;  // 16-byte chunks of a row; waves of a row
    float scale;
    uint16_t* out;
    int64_t ldo;
};
constexpr int kEmbedChunks = 2;  // 16-byte chunks of a thread

__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs p)
{
    const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, m = w / p.strips;
    if (m >= p.M) return;
    const int c0 = (int)(w - m * p.strips) * kWave * kEmbedChunks + (int)threadIdx.x % kWave;
    const int64_t id = p.ids[m];
    const bool some = id >= 0 && id < p.V;
    uint4 v[kEmbedChunks];
#pragma unroll
    for (int u = 0; u < kEmbedChunks; ++u) {
        const int c = c0 + kWave * u;
        const uint32_t fill = id >= p.V ? 0x7FC07FC0u : 0u;  // no such token: NaN; none: zeros
        v[u] = make_uint4(fill, fill, fill, fill);
        if (some && c < p.dc) v[u] = row_of(p.table, id, p.ldt)[c];
    }
#pragma unroll
    for (int u = 0; u < kEmbedChunks; ++u) {
        const int c = c0 + kWave * u;
        if (some && p.scale != 1.0f) {
            float f[8];
            unpack8(v[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= p.scale;
            v[u] = pack8(f);
        }
        if (c < p.dc) row_of(p.out, m, p.ldo)[c] = v[u];
    }
}

// ---- sorting the tokens --------------------------------------------------------------------------

__device__ inline uint32_t key_of(int64_t id, int64_t V) { return id >= 0 && id < V ? (uint32_t)id : kNoToken; }

struct SortArgs {
    const int64_t* ids;
    int64_t M, V;
    uint32_t *keys, *at;  // sorted within each chunk: ids and their positions
    int sort_blocks;
    uint4* table;  // to be filled with zeros by the other blocks
    int64_t ldt16, rows;
    int row16;  // 16-byte words of a row
};

// Blocks [0, sort_blocks) place 64 tokens of a chunk each; the others fill the gradient with zeros, one word a thread: short blocks
// that start in the order of their addresses write 6.8 TB/s, one to eight blocks a unit that go on by the grid's width 4.7 to 5.8
// (1 GiB; 4 KB blocks 157 us, 8 KB 168, 16 KB 170 to 176, past the caches 164, 256 blocks of 512 threads 186, 2048 of 256 226).
__global__ __launch_bounds__(kSortWaves* kWave) void embed_sort_kernel(const SortArgs p)
{
    if ((int)blockIdx.x >= p.sort_blocks) {
        const int64_t total = p.rows * p.row16, step = (int64_t)(gridDim.x - p.sort_blocks) * blockDim.x;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        int64_t i = (int64_t)(blockIdx.x - p.sort_blocks) * blockDim.x + threadIdx.x;
        if (p.ldt16 == p.row16) {
            for (; i < total; i += step) p.table[i] = zero;
        } else {
            for (; i < total; i += step) p.table[(i / p.row16) * p.ldt16 + i % p.row16] = zero;
        }
        return;
    }
    __shared__ uint32_t count[kSortWaves][kWave];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t mine = (int64_t)blockIdx.x * kSortBlock + lane, chunk = (int64_t)blockIdx.x * kSortBlock / kChunk * kChunk;
    const int64_t left = p.M - chunk, n = left < kChunk ? left : kChunk;
    const int own = (int)(mine - chunk);  // place in the chunk
    const uint32_t key = mine < p.M ? key_of(p.ids[mine], p.V) : kNoToken;
    // the 64-token groups of the chunk, dealt to the waves: those before this block's count equals too, those after do not
    uint32_t before = 0;
    const int groups = (int)((n + kWave - 1) / kWave), me = (int)((blockIdx.x * (int64_t)kSortBlock - chunk) / kWave);
    for (int g = wave; g < groups; g += kSortWaves) {
        const int64_t m = chunk + (int64_t)g * kWave + lane;
        const uint32_t other = m < chunk + n ? key_of(p.ids[m], p.V) : kNoToken;
        const int valid = (int)(n - (int64_t)g * kWave);  // of the group's tokens, maybe more than 64
        if (g < me) {
#pragma unroll 16
            for (int k = 0; k < kWave; ++k) before += (uint32_t)__builtin_amdgcn_readlane((int)other, k) <= key;
        } else if (g > me && valid >= kWave) {
#pragma unroll 16
            for (int k = 0; k < kWave; ++k) before += (uint32_t)__builtin_amdgcn_readlane((int)other, k) < key;
        } else {
            for (int k = 0; k < kWave && k < valid; ++k) {
                const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)other, k);
                before += o < key || (o == key && g * kWave + k < own);
            }
        }
    }
    count[wave][lane] = before;
    __syncthreads();
    if (wave == 0 && mine < p.M) {
        uint32_t r = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) r += count[w][lane];
        p.keys[chunk + r] = key, p.at[chunk + r] = (uint32_t)mine;
    }
}

// Sorted runs of `run` (a power of two) tokens to sorted runs of twice as many: a token's place is its own in its run and the number of those of
// the other run that come before it (positions are distinct and those of the left run come first, so equal ids keep their order).
__global__ __launch_bounds__(256) void embed_merge_kernel(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ at, uint32_t* __restrict__ out_keys,
                                                          uint32_t* __restrict__ out_at, int64_t M, int64_t run)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= M) return;
    const int64_t pair = i & -(2 * run), left = pair, right = pair + run;
    const bool in_left = i < right;
    const uint32_t key = keys[i];
    int64_t lo = in_left ? right : left, hi = in_left ? (right + run < M ? right + run : M) : right;
    const int64_t base = lo;
    if (lo > M) lo = hi = M;
    while (lo < hi) {  // the first that does not come before this token
        const int64_t mid = (lo + hi) / 2;
        const bool first = in_left ? keys[mid] < key : keys[mid] <= key;
        if (first) lo = mid + 1;
        else hi = mid;
    }
    const int64_t others = base > M ? 0 : lo - base;
    const int64_t to = pair + (in_left ? i - left : i - right) + others;
    out_keys[to] = key, out_at[to] = at[i];
}

// ---- the sums ------------------------------------------------------------------------------------

struct EmbedGradArgs {
    const uint32_t *keys, *at;  // sorted
    const uint16_t* dout;
    int64_t lddo, M;
    int dc, strips, piece;  // strips of 512 columns; tokens of a piece
    int64_t pieces;
    float scale;
    void* dtable;
    int64_t ldt;
    float* part;  // [piece][0: the run it begins with, if that began before; 1: the one it ends with, if that goes on][D]
};

template <bool F32>
__device__ inline void put_row(const EmbedGradArgs& p, uint32_t id, int c, const float* acc)
{
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = acc[j] * p.scale;
    if constexpr (F32) {
        float4* o = reinterpret_cast<float4*>(static_cast<float*>(p.dtable) + (int64_t)id * p.ldt) + 2 * c;
        o[0] = make_float4(f[0], f[1], f[2], f[3]), o[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        row_of(static_cast<uint16_t*>(p.dtable), id, p.ldt)[c] = pack8(f);
    }
}

template <bool F32>
__global__ __launch_bounds__(256) void embed_pieces_kernel(const EmbedGradArgs p)
{
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), piece = w / p.strips;
    if (piece >= p.pieces) return;
    const int c = (int)(w - piece * p.strips) * kWave + (int)threadIdx.x % kWave;
    const bool in = c < p.dc;
    const int64_t first = piece * p.piece, end = first + p.piece < p.M ? first + p.piece : p.M;
    uint32_t id = p.keys[first];
    if (id == kNoToken) return;  // so are all that follow
    const bool goes_on = end < p.M && p.keys[end] == p.keys[end - 1] && p.keys[end] != kNoToken;
    bool began_before = first > 0 && p.keys[first - 1] == id;
    float acc[8] = {};
    auto leave = [&](bool last) {
        if (!in) return;
        if (began_before || (last && goes_on)) {
            float4* o = reinterpret_cast<float4*>(p.part + ((piece * 2 + (began_before ? 0 : 1)) * p.dc + c) * 8);
            o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]), o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        } else {
            put_row<F32>(p, id, c, acc);
        }
    };
    constexpr int AHEAD = 8;
    for (int64_t i0 = first; i0 < end; i0 += AHEAD) {
        uint32_t k[AHEAD];
        uint4 v[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t i = i0 + a < end ? i0 + a : end - 1;
            k[a] = i0 + a < end ? p.keys[i] : kNoToken;
            v[a] = make_uint4(0, 0, 0, 0);
            if (k[a] != kNoToken && in) v[a] = load_once(row_of(p.dout, p.at[i], p.lddo) + c);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (k[a] == kNoToken) break;  // (uniform, as the ids are)
            if (k[a] != id) {
                leave(false);
                began_before = false, id = k[a];
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
            }
            float f[8];
            unpack8(v[a], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += f[j];
        }
    }
    leave(true);
}

// One wave for each piece and strip: if a run of tokens that goes on over the next pieces begins in this one, its sum.
template <bool F32>
__global__ __launch_bounds__(256) void embed_join_kernel(const EmbedGradArgs p)
{
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), piece = w / p.strips;
    const int64_t first = piece * p.piece, end = first + p.piece;
    if (piece >= p.pieces || end >= p.M) return;
    const uint32_t id = p.keys[end - 1];
    if (id == kNoToken || p.keys[end] != id) return;                          // ends here
    if (p.keys[first] == id && first > 0 && p.keys[first - 1] == id) return;  // began before
    const int lane = threadIdx.x % kWave, c = (int)(w - piece * p.strips) * kWave + lane;
    // how many of the next pieces begin with this id
    int64_t more = 0;
    for (;;) {
        const int64_t at = end + (more + lane) * p.piece;
        const uint64_t same = __ballot(at < p.M && p.keys[at < p.M ? at : 0] == id);
        if (~same) {
            more += __builtin_ctzll(~same);
            break;
        }
        more += kWave;
    }
    if (c >= p.dc) return;
    const float4* src = reinterpret_cast<const float4*>(p.part + ((piece * 2 + 1) * p.dc + c) * 8);
    float4 a = src[0], b = src[1];
    src = reinterpret_cast<const float4*>(p.part + ((piece + 1) * 2 * p.dc + c) * 8);
    const int64_t step = (int64_t)4 * p.dc;  // of float4: two rows of D
    constexpr int AHEAD = 16;
    for (int64_t k = 0; k < more; k += AHEAD) {
        float4 va[AHEAD], vb[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            va[u] = vb[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (k + u < more) va[u] = src[(k + u) * step], vb[u] = src[(k + u) * step + 1];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            a.x += va[u].x, a.y += va[u].y, a.z += va[u].z, a.w += va[u].w;
            b.x += vb[u].x, b.y += vb[u].y, b.z += vb[u].z, b.w += vb[u].w;
        }
    }
    const float acc[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    put_row<F32>(p, id, c, acc);
}

// ---- host ----------------------------------------------------------------------------------------

// Tokens of a piece: enough pieces to fill the chip with the waves of a few strips, and few enough that their sums of one id are
// joined in a moment.
static int piece_of(int64_t M)
{
    const int64_t n = (M + 1023) / 1024;
    return (int)(n < 8 ? 8 : n);
}
struct EmbedPlan {
    int piece;
    int64_t pieces;
    size_t list;   // bytes of a sorted list of words
    int lists;     // two for one chunk, two more to merge into
    size_t bytes;  // of the workspace
};
static EmbedPlan plan_embed(int64_t M, int64_t D)
{
    EmbedPlan e;
    e.piece = piece_of(M), e.pieces = (M + e.piece - 1) / e.piece;
    e.list = ((size_t)M * sizeof(uint32_t) + 255) / 256 * 256, e.lists = M > kChunk ? 4 : 2;
    e.bytes = kMinWorkspaceBytes + e.lists * e.list + (size_t)e.pieces * 2 * D * sizeof(float);
    return e;
}
// Enough for M tokens and for any number below: pieces get fewer where they get longer (9217 tokens have 922 of 10, 9216 have 1024 of
// 9), so their number is taken as its bound for all up to M, of 8 tokens each and 1024 in all.
static size_t embed_bytes(int64_t M, int64_t D)
{
    const EmbedPlan e = plan_embed(M, D);
    const int64_t eights = (M + 7) / 8, most = eights < 1024 ? eights : 1024;
    return e.bytes + (size_t)(most - e.pieces) * 2 * D * sizeof(float);
}

constexpr int64_t kEmbedMaxD = 1 << 20;
static bool bad_size(int64_t M, int64_t V, int64_t D) { return M < 0 || M > kEmbedMaxTokens || V < 0 || V > 0x7FFFFFFF || D < 0 || D > kEmbedMaxD || (D % 8); }
static bool bad_pitch(int64_t ld, int64_t D) { return ld < D || (ld % 8); }

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_embed_bwd_workspace_bytes(int64_t M, int64_t V, int64_t D)
{
    if (bad_size(M, V, D)) return kMinWorkspaceBytes;
    return embed_bytes(M, D);
}

f8_status f8_embed(const int64_t* ids, int64_t M, const void* table_bf16, int64_t ldt, int64_t V, int64_t D, float scale, void* out_bf16, int64_t ldo,
                   void* stream)
{
    if (bad_size(M, V, D) || !(scale - scale == 0.0f)) return F8_ERR_SHAPE;
    if (M != 0 && (!ids || !out_bf16 || (!table_bf16 && V != 0))) return F8_ERR_NULL;
    if (bad_pitch(ldt, D) || bad_pitch(ldo, D)) return F8_ERR_SHAPE;
    if (!aligned16(table_bf16) || !aligned16(out_bf16) || ((uintptr_t)ids & 7)) return F8_ERR_ALIGN;
    if (M > 0 && D > 0) {
        const int dc = (int)(D / 8), strips = (dc + kWave * kEmbedChunks - 1) / (kWave * kEmbedChunks);
        const int64_t blocks = (M * strips + 3) / 4;
        if (blocks > 0xFFFFFF) return F8_ERR_SHAPE;  // (a launch has less than 2^32 threads)
        embed_kernel<<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>({ids, (const uint16_t*)table_bf16, ldt, M, V, dc, strips, scale, (uint16_t*)out_bf16, ldo});
    }
    return last_launch_status();
}

f8_status f8_embed_bwd(const int64_t* ids, int64_t M, const void* dout_bf16, int64_t lddo, int64_t V, int64_t D, float scale, f8_dtype dtable_type,
                       void* dtable, int64_t ldt, void* workspace, size_t workspace_bytes_, void* stream)
{
    if ((int)dtable_type != F8_BF16 && (int)dtable_type != F8_F32) return F8_ERR_ENUM;
    if (bad_size(M, V, D) || !(scale - scale == 0.0f)) return F8_ERR_SHAPE;
    if ((V != 0 && !dtable) || (M != 0 && (!ids || !dout_bf16))) return F8_ERR_NULL;
    if (bad_pitch(lddo, D) || bad_pitch(ldt, D)) return F8_ERR_SHAPE;
    if (!aligned16(dout_bf16) || !aligned16(dtable) || !aligned16(workspace) || ((uintptr_t)ids & 7)) return F8_ERR_ALIGN;
    const EmbedPlan plan = plan_embed(M, D);
    if (M != 0 && (!workspace || workspace_bytes_ < plan.bytes)) return F8_ERR_WORKSPACE;
    const int dc = (int)(D / 8), strips = (dc + kWave - 1) / kWave;
    const int64_t blocks = (plan.pieces * strips + 3) / 4;
    if (V == 0 || D == 0) return last_launch_status();
    hipStream_t st = (hipStream_t)stream;
    const bool f32 = dtable_type == F8_F32;
    uint32_t* list[4];
    for (int i = 0; i < 4; ++i) list[i] = (uint32_t*)((char*)workspace + kMinWorkspaceBytes + (i < plan.lists ? i : 0) * plan.list);
    float* const part = (float*)((char*)workspace + kMinWorkspaceBytes + plan.lists * plan.list);

    const int row16 = (int)(D * (f32 ? 4 : 2) / 16), sort_blocks = (int)((M + kSortBlock - 1) / kSortBlock);
    const int64_t words = V * row16, fill = (words + kSortWaves * kWave - 1) / (kSortWaves * kWave);
    embed_sort_kernel<<<(unsigned)(sort_blocks + (fill < kMaxFillBlocks ? fill : kMaxFillBlocks)), kSortWaves * kWave, 0, st>>>(
        {ids, M, V, list[0], list[1], sort_blocks, (uint4*)dtable, ldt * (f32 ? 4 : 2) / 16, V, row16});
    if (M == 0) return last_launch_status();
    int from = 0;
    for (int64_t run = kChunk; run < M; run *= 2, from ^= 2)
        embed_merge_kernel<<<(unsigned)((M + 255) / 256), 256, 0, st>>>(list[from], list[from + 1], list[from ^ 2], list[(from ^ 2) + 1], M, run);
    const EmbedGradArgs a = {list[from], list[from + 1], (const uint16_t*)dout_bf16, lddo, M, dc, strips, plan.piece, plan.pieces, scale, dtable, ldt, part};
    (f32 ? embed_pieces_kernel<true> : embed_pieces_kernel<false>)<<<(unsigned)blocks, 256, 0, st>>>(a);
    if (plan.pieces > 1) (f32 ? embed_join_kernel<true> : embed_join_kernel<false>)<<<(unsigned)blocks, 256, 0, st>>>(a);
    return last_launch_status();
}

}  // extern "C"
