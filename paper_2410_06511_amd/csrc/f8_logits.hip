// From the logits of an output projection to the loss and back to the logits' gradient (which is the output gradient of a Float8
// linear), a row of V logits z = scale * logits per token:
//   p = softmax(z),  logp[t] = z_t - lse,  H = -sum p log p,  the k largest z with their log p;
//   dz_j = scale * (dlogp (1[j = t] - p_j) - dH p_j (log p_j + H))
// and distillation from a teacher's listed entries (id_k, q_k), with p_rest, q_rest the masses outside the list:
//   loss = sum_k q_k (log q_k - log p_k) [+ q_rest (log q_rest - log p_rest)]
//   dz_j = scale * (g (p_j - q_j) + the given token's term above) [for j outside the list q_j = q_rest s_j, where s is the softmax
//   of the logits outside the list alone].
// Bound by memory: one read of the logits forward (2 bytes an element), one read and one write backward (4 bytes).  8192 x 131072
// forward 314 us (6.8 TB/s), backward 783 (5.5); beside the loads stand about 9 instructions and an exponential an element, which keep
// the vector units busy for 79 % of the time, 92 % with alternatives and 94 % with a teacher's list and the rest (4096 x 131072 166 us).
// Softmax statistics are kept as (largest logit, log of the sum of exp(z - z_max)): a difference of two bf16 values is exact in
// fp32 where their ratio is below 2^16, so that p keeps its precision however large the logits are, which one number lse would not.
#include <float.h>

#include <type_traits>

#include "f8_device.hpp"
#include "f8_host.hpp"

namespace f8 {

// A block of 256 threads holds little enough that several share a compute unit and hide each other's selection, joins and ends
// (8192 x 32768 with 32 alternatives 111 us, with 512 threads 137); four loads a thread (two 116, eight 122).
constexpr int kLgThreads = 256;         // of a block of the forward
constexpr int kLgWaves = kLgThreads / kWave;
constexpr int kLgGradUnroll = 4;
constexpr int kLgUnroll = 4;            // 16-byte loads in flight a thread: the chunks of one step
constexpr int kLgSegCols = 131072;      // columns that a block takes at most
constexpr int kLgMaxSeg = 32;           // blocks that share a row, at most
constexpr int64_t kLgMaxCols = (int64_t)kLgSegCols * kLgMaxSeg;
constexpr int kLgMaxTop = 128;          // alternatives, and entries of a teacher's list
constexpr int kLgCandidates = 1024;     // elements that the selection ranks at once
constexpr int kLgGradBlocks = 2048;     // of the gradient: one partial maximum each (1024: 8192 x 131072 832 -> 867 us)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr uint32_t kNegInf2 = 0xFF80FF80u;
static_assert((size_t)kLgGradBlocks * sizeof(uint32_t) <= kMinWorkspaceBytes, "one partial maximum per block fits the minimum workspace");
static_assert(kLgMaxTop <= kLgThreads, "a thread an entry");
constexpr int kListWaves = kLgMaxTop / kWave;  // waves whose threads have an entry

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- statistics of a softmax, joined over lanes, waves and blocks -------------------------------

// m: largest logit seen (-FLT_MAX: none but -inf), s = sum e, e = exp(scale (z - m)); c = scale * log2(e);
// d: sum e log2(e) (ENT).
// Exponents end at kFar, where e is 0: differences of masked values (-inf, the type's lowest) would make 0 * inf.
constexpr float kFar = -1000.0f;
struct Stat {
    float m, s, d;
};
// v as seen from a larger maximum
template <bool ENT>
__device__ inline Stat raised(const Stat& v, float m, float c)
{
    const float g = fmaxf((v.m - m) * c, kFar), f = exp2_hw(g);
    return {m, v.s * f, ENT ? f * (v.d + v.s * g) : 0.0f};
}
template <bool ENT>
__device__ inline Stat join(const Stat& a, const Stat& b, float c)
{
    const float m = fmaxf(a.m, b.m);
    const Stat x = raised<ENT>(a, m, c), y = raised<ENT>(b, m, c);
    return {m, x.s + y.s, ENT ? x.d + y.d : 0.0f};
}
template <bool ENT>
__device__ inline Stat wave_join(Stat v, float c)
{
    return wave_all(v, [c](const Stat& a, const Stat& b) { return join<ENT>(a, b, c); });
}

// ---- order of logits -----------------------------------------------------------------------------

// bf16 bits -> 16 bits whose integer order is that of the values; both zeros alike, NaN as -inf (0x7F, the least)
__device__ inline uint32_t order16(uint32_t b)
{
    b = b == 0x8000u ? 0u : (b & 0x7FFFu) > 0x7F80u ? 0xFF80u : b;
    return b & 0x8000u ? ~b & 0xFFFFu : b | 0x8000u;
}
__device__ inline float order_value(uint32_t o) { return __uint_as_float((o & 0x8000u ? o & 0x7FFFu : ~o & 0xFFFFu) << 16); }
// elements in their order, the lower column first among equals
__device__ inline uint64_t element_key(uint32_t o, uint32_t col) { return (uint64_t)o << 32 | (uint32_t)~col; }
__device__ inline uint32_t key_column(uint64_t k) { return ~(uint32_t)k; }

// chunk c of a row; columns from V on read as -inf
template <bool ONCE>
__device__ inline uint4 load_logits(const uint4* row, int c, int V)
{
    uint4 v = ONCE ? load_once(row + c) : row[c];
    const int left = V - c * 8;
    if (left < 8) {
        uint32_t* w = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = left <= 2 * j ? kNegInf2 : left == 2 * j + 1 ? (w[j] & 0xFFFFu) | (kNegInf2 & 0xFFFF0000u) : w[j];
    }
    return v;
}

// ---- a teacher's list in LDS ----------------------------------------------------------------------

// The entries of one row that fall into a block's columns.  A chunk that holds some has a slot, the number of one of them; there its
// entries leave which elements they are and their weights.  The sweep leaves these chunks out, and the thread whose entry is the
// first element takes it: the same one whichever entry gave the slot its number, so that sums keep their order.
// (2048 x 32768 with 128 entries: forward 37 us, backward 53; adjacent tokens 32 and 48, 45 and 162 with a search among all entries.)
constexpr uint8_t kNoSlot = 0xFF;
template <bool WEIGHTS>
struct List {
    alignas(16) uint8_t slot[kLgSegCols / 8];
    alignas(16) float w[WEIGHTS ? kLgMaxTop : 1][8];  // by slot and element
    uint32_t mask[kLgMaxTop];                         // by slot
    int id[kLgMaxTop];                                // column, -1: none here
    float q[WEIGHTS ? kLgMaxTop : 1];
    uint32_t again;  // an id occurs twice
    __device__ bool marked(int lc) const { return slot[lc] != kNoSlot; }
};
static_assert(kLgMaxTop <= kNoSlot, "entries are numbered in a byte");
// Threads below K bring their entry (q: its weight), all THREADS call; chunks c0 .. c1 - 1.
template <int THREADS, bool WEIGHTS>
__device__ inline void list_fill(List<WEIGHTS>& L, int K, int64_t id, float q, int c0, int c1)
{
    const int k = threadIdx.x;
    const bool here = k < K && id >= (int64_t)c0 * 8 && id < (int64_t)c1 * 8;
    const int lc = here ? (int)(id >> 3) - c0 : 0, e = (int)(id & 7);
    for (int i = k; i < (c1 - c0 + 15) / 16; i += THREADS) reinterpret_cast<uint4*>(L.slot)[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
    if (k < kLgMaxTop) {
        L.id[k] = here ? (int)id : -1, L.mask[k] = 0;
        if constexpr (WEIGHTS) {
            L.q[k] = q;
            reinterpret_cast<float4*>(L.w[k])[0] = reinterpret_cast<float4*>(L.w[k])[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    }
    if (k == 0) L.again = 0;
    __syncthreads();
    if (here) L.slot[lc] = (uint8_t)k;  // (one of the chunk's entries stays)
    __syncthreads();
    if (here) {
        const int s = L.slot[lc];
        if (atomicOr(&L.mask[s], 1u << e) >> e & 1) L.again = 1;
        else if constexpr (WEIGHTS) L.w[s][e] = q;
    }
    __syncthreads();
}
// The chunk that this thread takes (-1: none): which of its elements are listed, and their weights (an id that occurs again
// counts with each of its weights, in their order).
template <bool WEIGHTS>
__device__ inline int list_chunk(const List<WEIGHTS>& L, int K, int c0, uint32_t* mask, float* w)
{
    const int k = threadIdx.x, id = k < K ? L.id[k] : -1;
    if (id < 0) return -1;
    const int s = L.slot[(id >> 3) - c0];
    *mask = L.mask[s];
    bool first = (id & 7) == __ffs(*mask) - 1;
    if constexpr (WEIGHTS) {
        const float4 a = reinterpret_cast<const float4*>(L.w[s])[0], b = reinterpret_cast<const float4*>(L.w[s])[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    if (L.again) {
        if constexpr (WEIGHTS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 0.0f;
        }
#pragma unroll 8
        for (int j = 0; j < K; ++j) {
            const int other = L.id[j];
            if (other == id && j < k) first = false;
            if constexpr (WEIGHTS) {
                if (other >> 3 == id >> 3) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] += e == (other & 7) ? L.q[j] : 0.0f;
                }
            }
        }
    }
    return first ? id >> 3 : -1;
}

// ---- forward ---------------------------------------------------------------------------------------

struct TeacherArgs {
    const int64_t* ids;  // [M, K], negative: no entry
    const float* logp;   // [M, K]
    int K, tail;
    float scale;
};
struct StatArgs {
    const uint16_t* logits;
    int64_t ld, M;
    int V, nseg, seg_chunks, top;
    float scale;
    const int64_t* targets;  // nullable
    float *stats, *logp, *entropy;
    int64_t* top_ids;
    float* top_logp;
    TeacherArgs t;
    float* loss;
    float4* part;        // per block of a shared row: (m, s, d, -), or (m, s) outside and inside the list
    uint64_t* part_top;  // and its elements
};

// a remainder that sums of fp32 probabilities do not tell from zero counts as none
constexpr double kNoRest = 0x1p-20;

// What a row's outputs need beside its statistics, read by one whole wave: ahead of the sweep, which hides these loads.
struct RowInputs {
    int64_t target;
    float zt;                          // its logit
    static constexpr int E = kLgMaxTop / kWave;
    float zk[E], lq[E];                // of the teacher's entries lane, lane + 64: the student's logit, the teacher's value
    bool has[E], wrong;
};
template <bool LIST>
__device__ inline RowInputs row_inputs(const StatArgs& a, int64_t row)
{
    const int lane = threadIdx.x & (kWave - 1);
    const uint16_t* z = a.logits + row * a.ld;
    RowInputs in = {};
    in.target = a.logp ? a.targets[row] : -1;
    if (in.target >= 0 && in.target < a.V) in.zt = __uint_as_float((uint32_t)z[in.target] << 16);
    if constexpr (LIST) {
#pragma unroll
        for (int e = 0; e < RowInputs::E; ++e) {
            const int k = lane + kWave * e;
            in.lq[e] = -INFINITY;
            if (k >= a.t.K) continue;
            const int64_t id = a.t.ids[row * a.t.K + k];
            const float t = a.t.logp[row * a.t.K + k];
            in.has[e] = id >= 0 && id < a.V;
            in.wrong |= id >= a.V;
            if (in.has[e]) in.zk[e] = __uint_as_float((uint32_t)z[id] << 16), in.lq[e] = t * a.t.scale;
        }
    }
    return in;
}

// What a row's outputs are, from its statistics; called by the same whole wave.
// With a teacher whose remainder is a class of its own v is of the logits outside the list and `listed` of those in it, each with its
// own largest: the remainder's log probability and gradient are finite however far below the list its logits lie.  The backward
// takes them as (largest outside the list, log of the sum of exponentials there over q_rest) in the row's last two numbers, the
// second +inf where there is nothing to subtract, -inf where the row has no term.
template <bool LIST>
__device__ inline void finish_row(const StatArgs& a, int64_t row, const RowInputs& in, Stat v, Stat listed)
{
    const int lane = threadIdx.x & (kWave - 1);
    constexpr int E = RowInputs::E;
    const Stat all = LIST && a.t.tail ? join<false>(v, listed, a.scale * kLog2e) : v;
    const float total = all.s;
    const bool none = total == 0.0f;  // every logit is -inf
    const float m = none ? -INFINITY : all.m, log_total = none ? -INFINITY : logf(total);
    if (lane == 0) {
        float* s = a.stats + row * (LIST ? 4 : 2);
        s[0] = m, s[1] = log_total;
        if (a.entropy) a.entropy[row] = none ? 0.0f : log_total - v.d * kLn2 / total;
        if (a.logp) {
            a.logp[row] = in.target < 0 ? 0.0f : in.target >= a.V ? NAN : none ? -INFINITY : (in.zt - m) * a.scale - log_total;
        }
    }
    if constexpr (LIST) {
        // the teacher's probabilities: given, or the softmax over its entries
        const float(&lq)[E] = in.lq;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) top = lq[e] > top || lq[e] != lq[e] ? lq[e] : top;
        double sum = 0.0;
        float norm = 0.0f;
        if (!a.t.tail) {
            top = wave_all(top, [](float x, float y) { return x != x ? x : x > y ? x : y; });  // (a NaN stays)
#pragma unroll
            for (int e = 0; e < E; ++e) sum += lq[e] == -INFINITY ? 0.0 : (double)expf(lq[e] - top);
            sum = wave_all(sum, [](double x, double y) { return x + y; });
            norm = sum == 0.0 ? 0.0f : top + logf((float)sum);
        }
        double loss = 0.0, mass = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float l = lq[e] - norm, q = lq[e] == -INFINITY ? 0.0f : expf(l);
            mass += q;
            if (q != 0.0f) loss += (double)q * (l - (none ? -INFINITY : (in.zk[e] - m) * a.scale - log_total));
        }
        loss = wave_all(loss, [](double x, double y) { return x + y; });
        mass = wave_all(mass, [](double x, double y) { return x + y; });
        float coef = none ? 0.0f : 1.0f;
        if (a.t.tail) {
            const double left = 1.0 - mass;
            const float q_rest = left < kNoRest ? 0.0f : (float)left;  // (a NaN stays)
            const bool rest = v.s != 0.0f;
            const double log_rest = rest ? logf(v.s / total) + ((double)v.m - m) * a.scale : -INFINITY;
            if (q_rest != 0.0f) loss += (double)q_rest * (logf(q_rest) - log_rest);
            coef = v.m, norm = mass != mass ? NAN : rest && q_rest != 0.0f ? logf(v.s / q_rest) : INFINITY;
        }
        // without entries (or weights to share out) there is no term, whatever the logits: marked for the backward by norm = -inf
        bool some = false;
#pragma unroll
        for (int e = 0; e < E; ++e) some |= in.has[e];
        if (a.t.tail ? !__any(some) : sum == 0.0) loss = coef = 0.0f, norm = -INFINITY;
        if (__any(in.wrong)) loss = coef = NAN, norm = a.t.tail ? NAN : 0.0f;
        if (lane == 0) {
            a.loss[row] = (float)loss;
            a.stats[row * 4 + 2] = coef, a.stats[row * 4 + 3] = norm;
        }
    }
}

// Places of n keys (all different) among themselves, by counting: emit(place, key) for the first K.  Where there are threads
// enough, 2 or 8 adjacent ones count for a key together.  keys has room for kRankPad more, which are set to 0 here (so that loads
// need no condition and go ahead together: 175 keys 23 000 cycles with one, now 6 000).
constexpr uint32_t kRankPad = 32;
template <int THREADS, class Emit>
__device__ inline void rank_keys(uint64_t* keys, uint32_t n, int K, Emit&& emit)
{
    if (threadIdx.x < kRankPad) keys[n + threadIdx.x] = 0;
    __syncthreads();
    const uint32_t lg = n <= THREADS / 8 ? 3 : n <= THREADS / 2 ? 1 : 0, part = threadIdx.x & ((1u << lg) - 1);
    for (uint32_t i0 = 0; i0 < n; i0 += THREADS >> lg) {
        const uint32_t i = i0 + (threadIdx.x >> lg);
        const uint64_t key = i < n ? keys[i] : 0;
        int rank = 0;
        for (uint32_t j = part; j < n && rank < K; j += 4u << lg) {
            uint64_t other[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) other[k] = keys[j + (k << lg)];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) rank += other[k] > key;
        }
        for (uint32_t off = 1; off < 1u << lg; off *= 2) rank += __shfl_xor(rank, off, kWave);
        if (i < n && part == 0 && rank < K) emit(rank, key);
    }
}

// Selection of a block's K largest elements.  A step's chunks of one thread (32 elements) leave their maximum in LDS, 2 bytes,
// and every thread knows its own largest.  The K-th largest of these bounds the search: K elements reach it, so the K best do, and
// they lie in steps whose maximum does.  Those are read again (about K, where the large elements are spread) and what reaches the
// bound is ranked by counting.
struct Select {
    uint64_t cand[kLgCandidates + kRankPad];
    uint16_t step[kLgCandidates];
    uint32_t best[kLgThreads];
    uint32_t bound, nstep, ncand;
};

// The largest value that at least K of the threads' maxima reach (every one of kLgThreads >= K has one, 0 if it saw nothing), or
// the first found that exactly K do.
__device__ inline uint32_t kth_best(const uint32_t* best, int K)
{
    const int lane = threadIdx.x & (kWave - 1);
    uint32_t k[kLgWaves], hi = 0, lo = 0;
#pragma unroll
    for (int i = 0; i < kLgWaves; ++i) k[i] = best[lane + kWave * i], hi = k[i] > hi ? k[i] : hi, lo = i == 0 || k[i] < lo ? k[i] : lo;
    hi = wave_all(hi, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    lo = wave_all(lo, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    while (lo < hi) {
        const uint32_t at = (lo + hi + 1) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kLgWaves; ++i) n += __popcll(__ballot(k[i] >= at));
        if (n >= K) lo = at;
        else hi = at - 1;
        if (n == K) break;
    }
    return lo;
}

// f(order, column) for the elements of chunk c that the row has
template <class F>
__device__ inline void each_element(const uint4* row, int c, int V, F&& f)
{
    const uint4 v = row[c];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c * 8 + j < V) f(order16(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu), (uint32_t)(c * 8 + j));
}

// The K largest in order: emit(rank, key).  smax: maxima by step * kLgThreads + thread; best: of this thread.
template <class Emit>
__device__ inline void block_top(const uint4* row, int c0, int c1, int V, int K, uint32_t best, const uint16_t* smax, Select& S, Emit&& emit)
{
    const int tid = threadIdx.x, steps = (c1 - c0 + kLgUnroll * kLgThreads - 1) / (kLgUnroll * kLgThreads);
    S.best[tid] = best;
    if (tid == 0) S.nstep = S.ncand = 0;
    __syncthreads();
    if (tid < kWave) {
        const uint32_t t = kth_best(S.best, K);
        if (tid == 0) S.bound = t;
    }
    __syncthreads();
    const uint32_t bound = S.bound;
    auto put = [&](uint32_t o, uint32_t col) {
        const uint32_t at = atomicAdd(&S.ncand, 1u);
        if (at < (uint32_t)kLgCandidates) S.cand[at] = element_key(o, col);
    };
    auto put_reaching = [&](int c) {  // what of a chunk reaches the bound, with one step of the counter
        const uint4 v = row[c];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            hits |= (uint32_t)(order16(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu) >= bound && c * 8 + j < V) << j;
        if (!hits) return;
        uint32_t at = atomicAdd(&S.ncand, (uint32_t)__popc(hits));
        for (; hits && at < (uint32_t)kLgCandidates; hits &= hits - 1, ++at) {
            const int j = __ffs(hits) - 1;
            const uint32_t pair = j < 4 ? (j < 2 ? v.x : v.y) : j < 6 ? v.z : v.w;
            S.cand[at] = element_key(order16(j & 1 ? pair >> 16 : pair & 0xFFFFu), (uint32_t)(c * 8 + j));
        }
    };
    if (best >= bound)
        for (int i = 0; i < steps; ++i)
            if (smax[i * kLgThreads + tid] >= bound && c0 + i * kLgUnroll * kLgThreads + tid < c1) {
                const uint32_t at = atomicAdd(&S.nstep, 1u);
                if (at < (uint32_t)kLgCandidates) S.step[at] = (uint16_t)(i * kLgThreads + tid);
            }
    __syncthreads();
    const uint32_t nstep = S.nstep;
    if (nstep <= (uint32_t)kLgCandidates) {
        for (uint32_t i = tid; i < nstep * kLgUnroll; i += kLgThreads) {
            const int st = S.step[i / kLgUnroll], c = c0 + (st / kLgThreads * kLgUnroll + (int)(i % kLgUnroll)) * kLgThreads + st % kLgThreads;
            if (c < c1) put_reaching(c);
        }
        __syncthreads();
    }
    uint32_t n = S.ncand;
    if (nstep > (uint32_t)kLgCandidates || n > (uint32_t)kLgCandidates) {
        // More equals of the bound than there is room for (rows of few values, or with little left by a mask): what is larger, and
        // then the equals from the row's front until there are enough.
        constexpr uint32_t kPiece = kWave * 8;  // elements of a wave's chunks
        __syncthreads();
        if (tid == 0) S.ncand = 0;
        __syncthreads();
        if (best > bound)
            for (int i = 0; i < steps; ++i)
                if (smax[i * kLgThreads + tid] > bound)
                    for (int u = 0; u < kLgUnroll; ++u) {
                        const int c = c0 + (i * kLgUnroll + u) * kLgThreads + tid;
                        if (c < c1) each_element(row, c, V, [&](uint32_t o, uint32_t col) { if (o > bound) put(o, col); });
                    }
        __syncthreads();
        n = S.ncand;
        __syncthreads();  // (every wave has the count before the first adds to it: the way on is one for the whole block)
        if (n <= kLgCandidates - kPiece) {
            for (int c = c0; c < c1 && n < (uint32_t)K; c += kWave) {
                if (tid < kWave && c + tid < c1) each_element(row, c + tid, V, [&](uint32_t o, uint32_t col) { if (o == bound) put(o, col); });
                __syncthreads();
                n = S.ncand;
                __syncthreads();
            }
        } else {
            // Large elements that share few threads: the K-th largest key itself, bit by bit.
            uint64_t t = 0;
            for (int bit = 47; bit >= 0; --bit) {
                const uint64_t at = t | (uint64_t)1 << bit;
                __syncthreads();
                if (tid == 0) S.ncand = 0;
                __syncthreads();
                uint32_t mine = 0;
                for (int i = 0; i < steps; ++i)
                    if (smax[i * kLgThreads + tid] >= (uint32_t)(at >> 32))
                        for (int u = 0; u < kLgUnroll; ++u) {
                            const int c = c0 + (i * kLgUnroll + u) * kLgThreads + tid;
                            if (c < c1) each_element(row, c, V, [&](uint32_t o, uint32_t col) { mine += element_key(o, col) >= at; });
                        }
                if (mine) atomicAdd(&S.ncand, mine);
                __syncthreads();
                if (S.ncand >= (uint32_t)K) t = at;
            }
            __syncthreads();
            if (tid == 0) S.ncand = 0;
            __syncthreads();
            for (int c = c0 + tid; c < c1; c += kLgThreads)
                each_element(row, c, V, [&](uint32_t o, uint32_t col) { if (element_key(o, col) >= t) put(o, col); });
            __syncthreads();
            n = S.ncand;
        }
    }
    rank_keys<kLgThreads>(S.cand, n, K, emit);
}

// One block takes one row, or one of nseg pieces of it.  Dynamic LDS (TOP): the steps' maxima.  LIST: with a teacher, TAIL: whose
// remainder is a class of its own, so that the statistics inside and outside the list are apart; those instances are held to the
// registers of six blocks a compute unit (84 without a bound, and five blocks: 4096 x 131072 167 -> 173 us, 8192 x 32768 102 -> 105).
template <bool ENT, bool TOP, bool LIST, bool TAIL, bool ONCE>
__global__ __launch_bounds__(kLgThreads, TAIL ? 6 : 1) void logits_stat_kernel(const StatArgs a)
{
    extern __shared__ uint16_t smax[];
    __shared__ Stat wave_stat[kLgWaves], wave_listed[kListWaves];
    __shared__ std::conditional_t<TOP, Select, int> sel;
    __shared__ std::conditional_t<TAIL, List<false>, int> list;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int chunks = (a.V + 7) / 8;
    const float c2 = a.scale * kLog2e;
    for (int64_t unit = blockIdx.x; unit < a.M * a.nseg; unit += gridDim.x) {
        const int64_t rowi = unit / a.nseg;
        const int seg = (int)(unit - rowi * a.nseg), c0 = seg * a.seg_chunks, c1 = c0 + a.seg_chunks < chunks ? c0 + a.seg_chunks : chunks;
        const uint4* row = reinterpret_cast<const uint4*>(a.logits + rowi * a.ld);
        Stat v = {-FLT_MAX, 0.0f, 0.0f}, listed = v;
        uint32_t best = 0;
        RowInputs in;
        if (a.nseg == 1 && wave == kLgWaves - 1) in = row_inputs<LIST>(a, rowi);
        uint4 w[kLgUnroll];
        auto request = [&](int c) {
#pragma unroll
            for (int u = 0; u < kLgUnroll; ++u)
                w[u] = c + u * kLgThreads < c1 ? load_logits<ONCE>(row, c + u * kLgThreads, a.V) : make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
        };
        if constexpr (TAIL) {
            const int64_t id = tid < a.t.K ? a.t.ids[rowi * a.t.K + tid] : -1;
            uint4 own = make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
            if (id >= (int64_t)c0 * 8 && id < (int64_t)c1 * 8) own = load_logits<false>(row, (int)(id >> 3), a.V);
            request(c0 + tid);
            list_fill<kLgThreads>(list, a.t.K, id, 0.0f, c0, c1);
            uint32_t mask;
            if (list_chunk(list, a.t.K, c0, &mask, nullptr) >= 0) {
                float z[8];
                unpack8(own, z);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool on = mask >> j & 1;
                    v.m = fmaxf(v.m, on ? -FLT_MAX : z[j]), listed.m = fmaxf(listed.m, on ? z[j] : -FLT_MAX);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool on = mask >> j & 1;
                    const float e = exp2_hw((z[j] - (on ? listed.m : v.m)) * c2);
                    v.s += on ? 0.0f : e, listed.s += on ? e : 0.0f;
                }
            }
            if (wave < kListWaves) {  // joined while the first step's loads are on their way
                const float m = wave_all(listed.m, [](float x, float y) { return fmaxf(x, y); });
                const float s = wave_all(raised<false>(listed, m, c2).s, [](float x, float y) { return x + y; });
                if (lane == 0) wave_listed[wave] = {m, s, 0.0f};
            }
        }
        for (int c = c0 + tid, step = 0; c < c1; c += kLgUnroll * kLgThreads, ++step) {
            if (!TAIL || step > 0) request(c);
            float z[kLgUnroll][8], m = -INFINITY;
#pragma unroll
            for (int u = 0; u < kLgUnroll; ++u) {
                unpack8(w[u], z[u]);
                if constexpr (TAIL)
                    if (c + u * kLgThreads < c1 && list.marked(c + u * kLgThreads - c0)) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) z[u][j] = -INFINITY;
                    }
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, z[u][j]);
            }
            if constexpr (TOP) {
                const uint32_t o = order16(__float_as_uint(m) >> 16);
                smax[step * kLgThreads + tid] = (uint16_t)o;
                best = o > best ? o : best;
            }
            v = raised<ENT>(v, fmaxf(v.m, m), c2);
#pragma unroll
            for (int u = 0; u < kLgUnroll; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float l = (z[u][j] - v.m) * c2, e = exp2_hw(l);
                    v.s += e;
                    if constexpr (ENT) v.d = __builtin_fmaf(e, fmaxf(l, kFar), v.d);
                }
        }
        v = wave_join<ENT>(v, c2);
        if (lane == 0) wave_stat[wave] = v;
        __syncthreads();
        v = wave_stat[0];
#pragma unroll
        for (int i = 1; i < kLgWaves; ++i) v = join<ENT>(v, wave_stat[i], c2);
        if constexpr (TAIL) {
            listed = wave_listed[0];
#pragma unroll
            for (int i = 1; i < kListWaves; ++i) listed = join<false>(listed, wave_listed[i], c2);
        }
        if (a.nseg > 1) {
            if (tid == 0) a.part[unit] = TAIL ? make_float4(v.m, v.s, listed.m, listed.s) : make_float4(v.m, v.s, v.d, 0.0f);
        }
        if constexpr (TOP) {
            const float log_total = logf(v.s);
            block_top(row, c0, c1, a.V, a.top, best, smax, sel, [&](int rank, uint64_t key) {
                if (a.nseg > 1) {
                    a.part_top[unit * a.top + rank] = key;
                } else {
                    a.top_ids[rowi * a.top + rank] = key_column(key);
                    a.top_logp[rowi * a.top + rank] = v.s == 0.0f ? -INFINITY : (order_value((uint32_t)(key >> 32)) - v.m) * a.scale - log_total;
                }
            });
        }
        if (a.nseg == 1 && wave == kLgWaves - 1) finish_row<LIST>(a, rowi, in, v, listed);  // (while the first waves rank)
        __syncthreads();  // LDS is used again
    }
}

// Rows that blocks shared: their statistics, and the best of their elements.
template <bool ENT, bool LIST>
__global__ __launch_bounds__(kLgThreads) void logits_join_kernel(const StatArgs a)
{
    extern __shared__ uint64_t cand[];  // [nseg * top + kRankPad]
    __shared__ uint32_t n;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const float c2 = a.scale * kLog2e;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const int keys = a.nseg * a.top;
        const uint64_t* lists = a.part_top + row * keys;
        constexpr int AHEAD = 4;  // keys that a thread has on their way beside the statistics
        RowInputs in;
        if (tid / kWave == kLgWaves - 1) in = row_inputs<LIST>(a, row);
        uint64_t mine[AHEAD], least = ~(uint64_t)0;
        Stat v = {-FLT_MAX, 0.0f, 0.0f}, listed = v;
        if (lane < a.nseg) {
            const float4 p = a.part[row * a.nseg + lane];
            v = {p.x, p.y, p.z};
            if (LIST && a.t.tail) listed = {p.z, p.w, 0.0f};
            // a key that K of the pieces' elements reach: the least of the pieces' (K / nseg)-th
            if (keys) least = lists[lane * a.top + (a.top + a.nseg - 1) / a.nseg - 1];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) mine[u] = tid + u * kLgThreads < keys ? lists[tid + u * kLgThreads] : 0;
        v = wave_join<ENT>(v, c2);
        if (LIST && a.t.tail) listed = wave_join<false>(listed, c2);
        if (keys) {
            least = wave_all(least, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
            if (tid == 0) n = 0;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (mine[u] >= least) cand[atomicAdd(&n, 1u)] = mine[u];
            for (int i = tid + AHEAD * kLgThreads; i < keys; i += kLgThreads) {
                const uint64_t key = lists[i];
                if (key >= least) cand[atomicAdd(&n, 1u)] = key;
            }
            __syncthreads();
            const float log_total = logf(v.s);
            rank_keys<kLgThreads>(cand, n, a.top, [&](int rank, uint64_t key) {
                a.top_ids[row * a.top + rank] = key_column(key);
                a.top_logp[row * a.top + rank] = v.s == 0.0f ? -INFINITY : (order_value((uint32_t)(key >> 32)) - v.m) * a.scale - log_total;
            });
        }
        if (tid / kWave == kLgWaves - 1) finish_row<LIST>(a, row, in, v, listed);  // (while the first waves rank)
        __syncthreads();
    }
}

// ---- backward ----------------------------------------------------------------------------------------

struct GradArgs {
    const uint16_t* logits;
    int64_t ld, M;
    int V, cols, nseg, seg_chunks;
    float scale;
    const int64_t* targets;
    const float *stats, *entropy, *d_logp, *d_entropy, *d_loss;
    TeacherArgs t;
    uint16_t* dlogits;
    int64_t ldd;
    uint32_t* partial;
};

template <int THREADS, bool ENT, bool LIST, bool ONCE>
__global__ __launch_bounds__(THREADS) void logits_grad_kernel(const GradArgs a)
{
    __shared__ uint32_t red[THREADS / kWave];
    __shared__ std::conditional_t<LIST, List<true>, int> list;
    const int tid = threadIdx.x;
    const int chunks = a.cols / 8, read = (a.V + 7) / 8;
    const float c2 = a.scale * kLog2e;
    uint32_t mag = 0;
    for (int64_t unit = blockIdx.x; unit < a.M * a.nseg; unit += gridDim.x) {
        const int64_t rowi = unit / a.nseg;
        const int seg = (int)(unit - rowi * a.nseg), c0 = seg * a.seg_chunks, c1 = c0 + a.seg_chunks < chunks ? c0 + a.seg_chunks : chunks;
        const uint4* row = reinterpret_cast<const uint4*>(a.logits + rowi * a.ld);
        uint4* out = reinterpret_cast<uint4*>(a.dlogits + rowi * a.ldd);
        const float* st = a.stats + rowi * (LIST ? 4 : 2);
        const float m = st[0], log2_total = st[1] * kLog2e;
        const int64_t target = a.targets ? a.targets[rowi] : -1;
        const float dlp = target < 0 || !a.d_logp ? 0.0f : target >= a.V ? NAN : a.d_logp[rowi] * a.scale;
        // dz = w (A + B log2 w), + dlp at the given token, w = exp2((z - mw) c2 - lw) = p; of listed entries p AL - their weight
        float A = -dlp, B = 0.0f, AL = 0.0f, mw = m, lw = log2_total;
        if constexpr (ENT) {
            const float dh = a.d_entropy[rowi] * a.scale;
            if (dh != 0.0f) A -= dh * a.entropy[rowi], B = -dh * kLn2;
        }
        float g = 0.0f;
        if constexpr (LIST) {
            g = st[3] == -INFINITY ? 0.0f : a.d_loss[rowi] * a.scale;  // (a row without entries has no term)
            AL = g - dlp;
            if (g != 0.0f) {
                if (!a.t.tail) {
                    A += g * st[2];
                } else if (st[3] == INFINITY) {
                    A = AL;
                } else {  // w is the rest's weight on this element, r = p / w = p_rest / q_rest (at most 2^20)
                    mw = st[2], lw = st[3] * kLog2e;
                    const float r = exp2_hw(__builtin_fmaf(mw - m, c2, lw) - log2_total);
                    A = g * (r - 1.0f) - dlp * r;
                }
            }
        }
        // nothing to hand back: no weight, or no logit that a change could move
        const bool zero = (A == 0.0f && B == 0.0f && dlp == 0.0f && g == 0.0f) || st[1] == -INFINITY;
        // chunk cu of the row, with the listed ones among its elements
        auto emit = [&](int cu, uint4 v, uint32_t mask, const float* q) {
            float z[8];
            unpack8(v, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool on = LIST && q && (mask >> j & 1);
                const float l2 = __builtin_fmaf(z[j] - (on ? m : mw), c2, -(on ? log2_total : lw)), w = exp2_hw(l2);
                z[j] = ENT ? w * __builtin_fmaf(B, fmaxf(l2, kFar), A) : on ? w * AL - q[j] : w * A;
            }
            if (cu == (int)(target >> 3)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] += j == (int)(target & 7) ? dlp : 0.0f;
            }
            const int left = a.V - cu * 8;
            if (left < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = j < left ? z[j] : 0.0f;
            }
            const uint4 o = make_uint4(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7]));
            mag = absmax_acc(mag, o);
            store_stream(out + cu, o);
        };
        uint4 w[kLgGradUnroll];
        auto request = [&](int c) {
#pragma unroll
            for (int u = 0; u < kLgGradUnroll; ++u) {
                const int cu = c + u * THREADS;
                w[u] = cu < c1 && cu < read && !zero ? load_logits<ONCE>(row, cu, a.V) : make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
            }
        };
        if constexpr (LIST) {
            if (!zero) {  // (alike for the whole block)
                int64_t id = -1;
                float t = 0.0f;
                uint4 own = make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
                if (tid < a.t.K) {
                    id = a.t.ids[rowi * a.t.K + tid];
                    if (id >= a.V) id = -1;
                    t = a.t.logp[rowi * a.t.K + tid];
                    if (id >= (int64_t)c0 * 8 && id < (int64_t)c1 * 8) own = load_logits<false>(row, (int)(id >> 3), a.V);
                }
                request(c0 + tid);
                const float norm = a.t.tail ? 0.0f : st[3];
                list_fill<THREADS>(list, a.t.K, id, id >= 0 && g != 0.0f ? g * expf(t * a.t.scale - norm) : 0.0f, c0, c1);
                uint32_t mask;
                float q[8];
                const int c = list_chunk(list, a.t.K, c0, &mask, q);
                if (c >= 0) emit(c, own, mask, q);
            }
        }
        for (int c = c0 + tid; c < c1; c += kLgGradUnroll * THREADS) {
            if (!LIST || zero || c != c0 + tid) request(c);
#pragma unroll
            for (int u = 0; u < kLgGradUnroll; ++u) {
                const int cu = c + u * THREADS;
                if (cu >= c1) break;
                if (zero || cu >= read) {
                    store_stream(out + cu, make_uint4(0, 0, 0, 0));
                    continue;
                }
                if constexpr (LIST)
                    if (list.marked(cu - c0)) continue;
                emit(cu, w[u], 0, nullptr);
            }
        }
        if constexpr (LIST) __syncthreads();  // LDS is used again
    }
    if (a.partial) {
        const uint32_t mx = block_max_u32<THREADS / kWave>(pk_collapse(mag), red);
        if (tid == 0) a.partial[blockIdx.x] = mx;
    }
}

// ---- host ---------------------------------------------------------------------------------------------

// Into how many pieces of how many chunks rows are cut: enough blocks for the chip where there are few rows, pieces of `least`
// chunks at least.
struct Split {
    int nseg, seg_chunks;
};
static Split split_rows(int64_t M, int64_t cols, int64_t blocks_wanted, int least)
{
    const int64_t chunks = (cols + 7) / 8, must = (cols + kLgSegCols - 1) / kLgSegCols;
    int64_t n = M > 0 ? blocks_wanted / M : 1;
    if (n > chunks / least) n = chunks / least;
    if (n > kLgMaxSeg) n = kLgMaxSeg;
    if (n < must) n = must;
    if (n < 1) n = 1;
    const int64_t per = (chunks + n - 1) / n;
    return {(int)((chunks + per - 1) / per), (int)per};
}
// The forward shares rows among blocks below two blocks a compute unit (more pieces cost more in the join than they bring: us with
// 512 / 1024 / 2048 blocks, 300 x 50001 with 64 alternatives 23 / 30 / 38, 512 x 50001 without 17.6 / 20.2 / 22.7), in pieces of a
// full step (of a chunk a thread at least: 100 x 8000 with 20 alternatives 14.8, so 9.5; 16 x 32768 16.2, so 13.3).
constexpr int64_t kLgBlocksWanted = 512;
// Loads past the caches.  Forward: from 1 GiB on, of which the backward would find little (8192 x 131072 357 -> 317 us, the backward
// unchanged; 6144 x 131072 275 -> 241, backward 533 -> 580; at the limit, 4096 x 131072, 188 -> 168 and 343 -> 374, with a teacher
// and the rest 193 -> 173 and 392 -> 404; below it 2048 x 131072 102 -> 93, but 188 -> 205).  Backward, the last to read: from
// 256 MiB on (4096 x 32768 85 -> 80, 2000 x 131072 with a teacher 211 -> 180; but 512 x 50001 21.9 -> 23.0).
constexpr int64_t kLgOnce = (int64_t)1 << 29, kLgGradOnce = (int64_t)1 << 27;

static size_t logits_part_bytes(int64_t M, int64_t V, int64_t top)
{
    const Split s = split_rows(M, V, kLgBlocksWanted, kLgUnroll * kLgThreads);
    return s.nseg > 1 ? (size_t)M * s.nseg * (sizeof(float4) + (size_t)top * sizeof(uint64_t)) : 0;
}

static bool bad_scale(float scale) { return !(scale > 0.0f) || !(scale * kLog2e <= FLT_MAX); }

static f8_status check_logits(const void* logits, int64_t ld, int64_t M, int64_t V, float scale, const void* stats)
{
    if (M != 0 && (!logits || !stats)) return F8_ERR_NULL;  // (without rows there is nothing that pointers point to)
    if (M < 0 || M > 0x7FFFFFFF || V < 1 || V > kLgMaxCols || ld < V || (ld % 8) || ld > 0x7FFFFFFF || bad_scale(scale)) return F8_ERR_SHAPE;
    if (!aligned16(logits)) return F8_ERR_ALIGN;
    return F8_OK;
}

static f8_status check_teacher(int64_t M, const int64_t* ids, const float* logp, int64_t K, int tail, float scale)
{
    if (M != 0 && (!ids || !logp)) return F8_ERR_NULL;
    if (tail != 0 && tail != 1) return F8_ERR_ENUM;
    if (K < 1 || K > kLgMaxTop || bad_scale(scale) || (tail && scale != 1.0f)) return F8_ERR_SHAPE;
    return F8_OK;
}

template <bool LIST>
static f8_status launch_stats(StatArgs& a, void* ws, size_t ws_bytes, hipStream_t st)
{
    if (a.M == 0) return F8_OK;
    const Split s = split_rows(a.M, a.V, kLgBlocksWanted, kLgUnroll * kLgThreads);
    a.nseg = s.nseg, a.seg_chunks = s.seg_chunks;
    if (a.nseg > 1) {
        if (!ws || ws_bytes < logits_part_bytes(a.M, a.V, a.top)) return F8_ERR_WORKSPACE;
        if (!aligned16(ws)) return F8_ERR_ALIGN;
        a.part = (float4*)ws;
        a.part_top = (uint64_t*)(a.part + a.M * a.nseg);
    }
    const int64_t units = a.M * a.nseg;
    const unsigned blocks = (unsigned)(units < (1 << 20) ? units : (1 << 20));
    const bool once = a.M * a.V >= kLgOnce;
    constexpr int kStep = kLgUnroll * kLgThreads;
    const size_t lds = a.top ? (size_t)(a.seg_chunks + kStep - 1) / kStep * kLgThreads * sizeof(uint16_t) : 0;
    if constexpr (LIST) {
        const auto kernel = a.t.tail ? (once ? logits_stat_kernel<false, false, true, true, true> : logits_stat_kernel<false, false, true, true, false>)
                                     : (once ? logits_stat_kernel<false, false, true, false, true> : logits_stat_kernel<false, false, true, false, false>);
        kernel<<<blocks, kLgThreads, lds, st>>>(a);
    } else {
        const auto kernel = a.top ? (a.entropy ? logits_stat_kernel<true, true, false, false, false> : logits_stat_kernel<false, true, false, false, false>)
                            : once ? (a.entropy ? logits_stat_kernel<true, false, false, false, true> : logits_stat_kernel<false, false, false, false, true>)
                                   : (a.entropy ? logits_stat_kernel<true, false, false, false, false> : logits_stat_kernel<false, false, false, false, false>);
        kernel<<<blocks, kLgThreads, lds, st>>>(a);
    }
    if (a.nseg > 1) {
        const unsigned rows = (unsigned)(a.M < (1 << 20) ? a.M : (1 << 20));
        const auto kernel = a.entropy ? logits_join_kernel<true, LIST> : logits_join_kernel<false, LIST>;
        kernel<<<rows, kLgThreads, ((size_t)a.nseg * a.top + kRankPad) * sizeof(uint64_t), st>>>(a);
    }
    return last_launch_status();
}

template <bool ENT, bool LIST>
static f8_status launch_grad(GradArgs& a, float* amax, void* ws, hipStream_t st)
{
    int nb = 0;
    if (a.M > 0) {
        // Blocks of 1024 threads where there are many long rows (8192 x 131072 819 -> 788 us, 8192 x 32768 168 -> 158; few rows lose:
        // 300 x 131072 36 -> 41, 777 x 50001 44 -> 52), with a teacher, whose list only two such blocks a compute unit set up, where
        // they are three times as long (4096 x 131072 420 -> 409, 3000 x 100000 230 -> 228; 4096 x 65536 192 -> 200, 8192 x 32768
        // 182 -> 221).  Else of 512, in pieces of a full step, or with a teacher of a quarter of the blocks, as every piece sets up
        // the list (64 x 131072 with 64 entries 19.5 -> 12.7, 300 x 50001 23 -> 18), but in as many as leave 4096 chunks to each
        // (600 x 131072 75 -> 63, 300 x 131072 34 -> 32; leaving 2048 or 8192: 62, 70 and 33, 35).
        Split s = split_rows(a.M, a.cols, kLgGradBlocks / 2, 1024);
        const bool wide = s.seg_chunks >= (LIST ? 3 : 1) * kLgGradUnroll * 1024 && a.M * s.nseg >= kLgGradBlocks;
        if (!wide) s = split_rows(a.M, a.cols, kLgGradBlocks, LIST ? 4096 : kLgGradUnroll * 512);
        if (LIST && !wide) {
            const Split quarter = split_rows(a.M, a.cols, kLgGradBlocks / 4, 512);
            if (quarter.nseg > s.nseg) s = quarter;
        }
        a.nseg = s.nseg, a.seg_chunks = s.seg_chunks;
        a.partial = amax ? (uint32_t*)ws : nullptr;
        const int64_t units = a.M * a.nseg;
        nb = (int)(units < kLgGradBlocks ? units : kLgGradBlocks);
        const bool once = a.M * a.V >= kLgGradOnce;
        const auto kernel = wide ? (once ? logits_grad_kernel<1024, ENT, LIST, true> : logits_grad_kernel<1024, ENT, LIST, false>)
                                 : (once ? logits_grad_kernel<512, ENT, LIST, true> : logits_grad_kernel<512, ENT, LIST, false>);
        kernel<<<nb, wide ? 1024 : 512, 0, st>>>(a);
    }
    if (amax) amax_final((const uint32_t*)ws, nb, amax, st);
    return last_launch_status();
}

static f8_status check_grad(int64_t M, int64_t V, const void* dlogits, int64_t ldd, int64_t cols, const float* amax, const void* ws, size_t ws_bytes)
{
    if (M != 0 && !dlogits) return F8_ERR_NULL;
    if (cols < V || (cols % 8) || cols > kLgMaxCols || ldd < cols || (ldd % 8) || ldd > 0x7FFFFFFF) return F8_ERR_SHAPE;
    if (!aligned16(dlogits)) return F8_ERR_ALIGN;
    if (amax && (!ws || ws_bytes < kMinWorkspaceBytes)) return F8_ERR_WORKSPACE;
    return F8_OK;
}

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_logits_workspace_bytes(int64_t M, int64_t V, int64_t top_k)
{
    size_t n = M > 0 && V > 0 && V <= kLgMaxCols && top_k >= 0 && top_k <= kLgMaxTop ? logits_part_bytes(M, V, top_k) : 0;
    if (n < kMinWorkspaceBytes) n = kMinWorkspaceBytes;
    return (n + 255) / 256 * 256;
}

f8_status f8_token_logprobs(const void* logits_bf16, int64_t ld, int64_t M, int64_t V, float scale, const int64_t* targets, float* stats, float* logp,
                            float* entropy, int64_t top_k, int64_t* top_ids, float* top_logp, void* workspace, size_t workspace_bytes_, void* stream)
{
    f8_status s = check_logits(logits_bf16, ld, M, V, scale, stats);
    if (s != F8_OK) return s;
    if (M != 0 && ((logp != nullptr) != (targets != nullptr) || (top_k > 0 && (!top_ids || !top_logp)))) return F8_ERR_NULL;
    if (top_k < 0 || top_k > kLgMaxTop || top_k > V) return F8_ERR_SHAPE;
    StatArgs a = {};
    a.logits = (const uint16_t*)logits_bf16, a.ld = ld, a.M = M, a.V = (int)V, a.top = (int)top_k, a.scale = scale;
    a.targets = targets, a.stats = stats, a.logp = logp, a.entropy = entropy, a.top_ids = top_ids, a.top_logp = top_logp;
    return launch_stats<false>(a, workspace, workspace_bytes_, (hipStream_t)stream);
}

f8_status f8_token_logprobs_bwd(const void* logits_bf16, int64_t ld, int64_t M, int64_t V, float scale, const int64_t* targets, const float* stats,
                                const float* entropy, const float* d_logp, const float* d_entropy, void* dlogits_bf16, int64_t ldd, int64_t cols,
                                float* amax_d, void* workspace, size_t workspace_bytes_, void* stream)
{
    f8_status s = check_logits(logits_bf16, ld, M, V, scale, stats);
    if (s != F8_OK) return s;
    if (M != 0 && ((d_logp != nullptr) != (targets != nullptr) || (d_entropy && !entropy) || (!d_logp && !d_entropy))) return F8_ERR_NULL;
    if ((s = check_grad(M, V, dlogits_bf16, ldd, cols, amax_d, workspace, workspace_bytes_)) != F8_OK) return s;
    GradArgs a = {};
    a.logits = (const uint16_t*)logits_bf16, a.ld = ld, a.M = M, a.V = (int)V, a.cols = (int)cols, a.scale = scale, a.targets = targets;
    a.stats = stats, a.entropy = entropy, a.d_logp = d_logp, a.d_entropy = d_entropy, a.dlogits = (uint16_t*)dlogits_bf16, a.ldd = ldd;
    return d_entropy ? launch_grad<true, false>(a, amax_d, workspace, (hipStream_t)stream)
                     : launch_grad<false, false>(a, amax_d, workspace, (hipStream_t)stream);
}

f8_status f8_distill(const void* logits_bf16, int64_t ld, int64_t M, int64_t V, float scale, const int64_t* teacher_ids, const float* teacher_logp, int64_t K,
                     int tail, float teacher_scale, const int64_t* targets, float* stats, float* loss, float* logp, void* workspace,
                     size_t workspace_bytes_, void* stream)
{
    f8_status s = check_logits(logits_bf16, ld, M, V, scale, stats);
    if (s != F8_OK) return s;
    if ((s = check_teacher(M, teacher_ids, teacher_logp, K, tail, teacher_scale)) != F8_OK) return s;
    if (M != 0 && (!loss || (logp != nullptr) != (targets != nullptr))) return F8_ERR_NULL;
    StatArgs a = {};
    a.logits = (const uint16_t*)logits_bf16, a.ld = ld, a.M = M, a.V = (int)V, a.scale = scale;
    a.targets = targets, a.stats = stats, a.logp = logp, a.t = {teacher_ids, teacher_logp, (int)K, tail, teacher_scale}, a.loss = loss;
    return launch_stats<true>(a, workspace, workspace_bytes_, (hipStream_t)stream);
}

f8_status f8_distill_bwd(const void* logits_bf16, int64_t ld, int64_t M, int64_t V, float scale, const int64_t* teacher_ids, const float* teacher_logp, int64_t K,
                         int tail, float teacher_scale, const int64_t* targets, const float* stats, const float* d_loss, const float* d_logp,
                         void* dlogits_bf16, int64_t ldd, int64_t cols, float* amax_d, void* workspace, size_t workspace_bytes_, void* stream)
{
    f8_status s = check_logits(logits_bf16, ld, M, V, scale, stats);
    if (s != F8_OK) return s;
    if ((s = check_teacher(M, teacher_ids, teacher_logp, K, tail, teacher_scale)) != F8_OK) return s;
    if (M != 0 && (!d_loss || (d_logp != nullptr) != (targets != nullptr))) return F8_ERR_NULL;
    if ((s = check_grad(M, V, dlogits_bf16, ldd, cols, amax_d, workspace, workspace_bytes_)) != F8_OK) return s;
    GradArgs a = {};
    a.logits = (const uint16_t*)logits_bf16, a.ld = ld, a.M = M, a.V = (int)V, a.cols = (int)cols, a.scale = scale, a.targets = targets;
    a.stats = stats, a.d_loss = d_loss, a.d_logp = d_logp, a.t = {teacher_ids, teacher_logp, (int)K, tail, teacher_scale};
    a.dlogits = (uint16_t*)dlogits_bf16, a.ldd = ldd;
    return launch_grad<false, true>(a, amax_d, workspace, (hipStream_t)stream);
}

}  // extern "C"
