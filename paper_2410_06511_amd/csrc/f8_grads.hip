// The norm of many gradients together, and their scaling to a largest norm, between a step's backward and its update:
//   norm = sqrt(sum over all tensors of x^2) (or the largest |x|),   out = x min(1, most / (norm + 1e-6)).
// Bound by memory: the norm reads every element once, the scaling reads and writes it.  Squares and sums are taken in fp64: the
// square of a bf16 or fp32 value is exact there and cannot overflow or vanish (fp32 loses gradients below 1e-19 and above 1e19),
// at a quarter of the rate that the memory leaves room for.
// One 8B block's gradients, 436 MB, us: norm 69 (6.3 TB/s), scaling 150 (5.8 TB/s); 216 tensors of 24 smaller blocks, 300 MB: 61 and 110.
// The tensors' addresses and sizes come as kernel arguments, kTensors to a launch; a block has a range of the steps of kStep
// elements of all of a launch's tensors.  Partial sums are added in a fixed order.
#include "f8_device.hpp"
#include "f8_host.hpp"

namespace f8 {

constexpr int kTensors = 128, kFewTensors = 16;  // of a launch: 3.6 KB of arguments, or half a KB
constexpr int kGradThreads = 256;
constexpr int kGradUnroll = 4;
constexpr int kStep = kGradThreads * 8 * kGradUnroll;  // elements
constexpr int kGradBlocks = 2048;  // of the norm: one partial sum each
constexpr uint32_t kClipBlocks = 16384;
// Lists larger than the last cache are loaded past the caches: what is read would be gone before it is wanted again, and what was
// written before has to leave.  Norm and scaling of 512 MB 296 -> 275 us, of 256 MB 149 -> 125, one 8B block 235 -> 220; of 192 MB
// in place 95 -> 105 (apart 104 -> 95), of 64 MB 37 -> 40.
constexpr int64_t kOnceBytes = (int64_t)1 << 28;

template <int CAP>
struct TensorList {
    const void* in[CAP];
    void* out[CAP];
    int64_t n[CAP];                     // elements
    uint32_t first[CAP + 1];            // the tensors' first steps; the number of steps
    uint32_t f32[(CAP + 31) / 32];      // bit i: tensor i holds fp32
    int count;
};

// f(tensor, first element) for every gridDim-th of the steps: the first one's tensor by bisection (the last whose first step is not
// behind it), then the next ones; all of it in scalar registers.  (Neighbouring steps for a block read slower: the scaling of one
// 8B block's gradients 151 -> 172 us.  From the last step on, which the norm has read latest, nothing is gained: 153.)
template <int CAP, class F>
__device__ inline void each_step(const TensorList<CAP>& l, F&& f)
{
    const uint32_t steps = l.first[l.count];
    int t = 0, hi = l.count;
    while (hi - t > 1) {
        const int mid = (t + hi) / 2;
        if (l.first[mid] <= blockIdx.x) t = mid;
        else hi = mid;
    }
    for (uint32_t step = blockIdx.x; step < steps; step += gridDim.x) {
        while (step >= l.first[t + 1]) ++t;
        f(t, (int64_t)(step - l.first[t]) * kStep);
    }
}

// Tensors lie on any element: loads and stores of eight are those of the element's alignment (the memory takes them, two lines
// instead of one now and then).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
__device__ inline uint4 load_any(const void* p) { return __builtin_bit_cast(uint4, (u32x4)*static_cast<const u32x4_any*>(p)); }
__device__ inline void store_any(void* p, uint4 v) { *static_cast<u32x4_any*>(p) = __builtin_bit_cast(u32x4, v); }

__device__ inline uint4 load_any_once(const void* p) { return __builtin_bit_cast(uint4, (u32x4)__builtin_nontemporal_load(static_cast<const u32x4_any*>(p))); }

struct Eight {
    uint4 a, b;  // b: fp32 only
};
template <bool F32>
__device__ inline void widen(const Eight& e, float* f)
{
    if constexpr (F32) {
        f[0] = __uint_as_float(e.a.x), f[1] = __uint_as_float(e.a.y), f[2] = __uint_as_float(e.a.z), f[3] = __uint_as_float(e.a.w);
        f[4] = __uint_as_float(e.b.x), f[5] = __uint_as_float(e.b.y), f[6] = __uint_as_float(e.b.z), f[7] = __uint_as_float(e.b.w);
    } else {
        unpack8(e.a, f);
    }
}
template <bool F32, bool ONCE = false>
__device__ inline Eight load8(const void* in, int64_t i)  // elements i .. i + 7
{
    const auto load = [](const char* p) { return ONCE ? load_any_once(p) : load_any(p); };
    const char* const at = static_cast<const char*>(in) + i * (F32 ? 4 : 2);
    return {load(at), F32 ? load(at + 16) : make_uint4(0, 0, 0, 0)};
}
template <bool F32>
__device__ inline float load1(const void* in, int64_t i)
{
    return F32 ? static_cast<const float*>(in)[i] : bf16_lo(static_cast<const uint16_t*>(in)[i]);
}

// ---- norm ----------------------------------------------------------------------------------------

// MAX: magnitudes by their bits, so that a NaN is larger than everything.
template <bool MAX>
struct Norm {
    double s[2] = {0.0, 0.0};
    uint32_t m = 0;
    __device__ void add(float v, int k)
    {
        if constexpr (MAX) {
            const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
            m = b > m ? b : m;
        } else {
            s[k & 1] = __builtin_fma((double)v, (double)v, s[k & 1]);
        }
    }
    __device__ double value() const { return MAX ? (double)__uint_as_float(m) : s[0] + s[1]; }
};
__device__ inline double join(double a, double b, bool max) { return max ? (a != a || a > b ? a : b) : a + b; }

template <bool MAX>
__device__ inline double block_join(double v, double* red)
{
    for (int off = 32; off >= 1; off >>= 1) v = join(v, __shfl_xor(v, off, kWave), MAX);
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < (int)blockDim.x / kWave; ++w) v = join(v, red[w], MAX);
    return v;
}

template <bool MAX, bool F32, bool ONCE>
__device__ inline void norm_step(const void* in, int64_t n, int64_t at, Norm<MAX>& norm)
{
    if (at + kStep <= n) {
        Eight e[kGradUnroll];
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) e[u] = load8<F32, ONCE>(in, at + (u * kGradThreads + (int)threadIdx.x) * 8);
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) {
            float f[8];
            widen<F32>(e[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) norm.add(f[j], j);
        }
    } else {
        for (int64_t i = at + (int)threadIdx.x * 8; i < n; i += kGradThreads * 8) {
            if (i + 8 <= n) {
                float f[8];
                widen<F32>(load8<F32>(in, i), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) norm.add(f[j], j);
            } else {
                for (int64_t k = i; k < n; ++k) norm.add(load1<F32>(in, k), 0);
            }
        }
    }
}

template <bool MAX, bool ONCE, int CAP>
__global__ __launch_bounds__(kGradThreads) void grad_norm_kernel(const TensorList<CAP> l, double* __restrict__ part)
{
    __shared__ double red[kGradThreads / kWave];
    Norm<MAX> norm;
    each_step(l, [&](int t, int64_t at) {
        if (l.f32[t / 32] >> (t % 32) & 1) norm_step<MAX, true, ONCE>(l.in[t], l.n[t], at, norm);
        else norm_step<MAX, false, ONCE>(l.in[t], l.n[t], at, norm);
    });
    const double v = block_join<MAX>(norm.value(), red);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

template <bool MAX>
__global__ __launch_bounds__(1024) void grad_norm_final_kernel(const double* __restrict__ part, int64_t n, float* norm, double* sum)
{
    __shared__ double red[1024 / kWave];
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) v = join(v, part[i], MAX);
    v = block_join<MAX>(v, red);
    if (threadIdx.x == 0) {
        if (norm) norm[0] = (float)(MAX ? v : __builtin_sqrt(v));
        if (sum) sum[0] = v;
    }
}

// ---- scaling -------------------------------------------------------------------------------------

template <bool F32, bool ONCE>
__device__ inline void clip_step(const void* in, void* out, int64_t n, int64_t at, float factor)
{
    const auto put = [&](const Eight& e, int64_t i) {
        char* o = static_cast<char*>(out) + i * (F32 ? 4 : 2);
        if (factor == 1.0f) {  // the same bits
            store_any(o, e.a);
            if (F32) store_any(o + 16, e.b);
            return;
        }
        float f[8];
        widen<F32>(e, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= factor;
        if constexpr (F32) {
            store_any(o, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
            store_any(o + 16, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
        } else {
            store_any(o, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
        }
    };
    if (at + kStep <= n) {
        Eight e[kGradUnroll];
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) e[u] = load8<F32, ONCE>(in, at + (u * kGradThreads + (int)threadIdx.x) * 8);
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) put(e[u], at + (u * kGradThreads + (int)threadIdx.x) * 8);
    } else {
        for (int64_t i = at + (int)threadIdx.x * 8; i < n; i += kGradThreads * 8) {
            if (i + 8 <= n) {
                put(load8<F32>(in, i), i);
            } else {
                for (int64_t k = i; k < n; ++k) {
                    if constexpr (F32) {
                        const float v = static_cast<const float*>(in)[k];
                        static_cast<float*>(out)[k] = factor == 1.0f ? v : v * factor;
                    } else {
                        const uint16_t v = static_cast<const uint16_t*>(in)[k];
                        static_cast<uint16_t*>(out)[k] = factor == 1.0f ? v : (uint16_t)pack_bf16(bf16_lo(v) * factor, 0.0f);
                    }
                }
            }
        }
    }
}

template <bool ONCE, int CAP>
__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(const TensorList<CAP> l, const float* __restrict__ norm, float most)
{
    float factor = most / (norm[0] + 1e-6f);
    factor = factor > 1.0f ? 1.0f : factor;  // (a NaN stays one)
    each_step(l, [&](int t, int64_t at) {
        if (factor == 1.0f && l.in[t] == l.out[t]) return;
        if (l.f32[t / 32] >> (t % 32) & 1) clip_step<true, ONCE>(l.in[t], l.out[t], l.n[t], at, factor);
        else clip_step<false, ONCE>(l.in[t], l.out[t], l.n[t], at, factor);
    });
}

// ---- host ----------------------------------------------------------------------------------------

constexpr int64_t kMaxElements = (int64_t)1 << 40;  // of a tensor

static f8_status check_list(const f8_tensor* list, int64_t count)
{
    if (count < 0) return F8_ERR_SHAPE;
    if (count && !list) return F8_ERR_NULL;
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].type != F8_BF16 && list[i].type != F8_F32) return F8_ERR_ENUM;
        if (list[i].n < 0 || list[i].n > kMaxElements) return F8_ERR_SHAPE;
        if (list[i].n && !list[i].data) return F8_ERR_NULL;
        if ((uintptr_t)list[i].data & (list[i].type == F8_F32 ? 3 : 1)) return F8_ERR_ALIGN;
    }
    return F8_OK;
}

static int64_t element_bytes(const f8_tensor& t) { return t.type == F8_F32 ? 4 : 2; }
static int64_t list_bytes(const f8_tensor* list, int64_t count)
{
    int64_t bytes = 0;
    for (int64_t i = 0; i < count && bytes < kOnceBytes; ++i) bytes += list[i].n * element_bytes(list[i]);
    return bytes;
}

// The list in launches of at most CAP tensors and 2^31 steps: f(TensorList, steps).
template <int CAP, class F>
static void for_launches(const f8_tensor* in, const f8_tensor* out, int64_t count, F&& f)
{
    TensorList<CAP> l;
    const auto clear = [&] {
        l.count = 0, l.first[0] = 0;
        for (auto& w : l.f32) w = 0;
    };
    clear();
    for (int64_t i = 0; i < count; ++i) {
        if (in[i].n == 0) continue;
        const uint32_t steps = (uint32_t)((in[i].n + kStep - 1) / kStep);
        if (l.count == CAP || (uint64_t)l.first[l.count] + steps > 0x7FFFFFFFu) f(l), clear();
        l.in[l.count] = in[i].data, l.out[l.count] = out ? out[i].data : nullptr, l.n[l.count] = in[i].n;
        if (in[i].type == F8_F32) l.f32[l.count / 32] |= 1u << (l.count % 32);
        l.first[l.count + 1] = l.first[l.count] + steps;
        ++l.count;
    }
    if (l.count) f(l);
}
static unsigned grad_blocks(uint32_t steps) { return steps < kGradBlocks ? steps : kGradBlocks; }
// Blocks of all launches: as for_launches deals the tensors out.
static int64_t all_blocks(const f8_tensor* list, int64_t count)
{
    int64_t blocks = 0, steps = 0, tensors = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].n == 0) continue;
        const int64_t more = (list[i].n + kStep - 1) / kStep;
        if (tensors == kTensors || steps + more > 0x7FFFFFFF) blocks += grad_blocks((uint32_t)steps), steps = tensors = 0;
        steps += more, ++tensors;
    }
    return blocks + grad_blocks((uint32_t)steps);
}
static size_t norm_bytes(const f8_tensor* list, int64_t count)
{
    const size_t bytes = (size_t)all_blocks(list, count) * sizeof(double);
    return bytes < kMinWorkspaceBytes ? kMinWorkspaceBytes : bytes;
}

}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_grad_norm_workspace_bytes(const f8_tensor* list, int64_t count)
{
    return check_list(list, count) == F8_OK ? norm_bytes(list, count) : kMinWorkspaceBytes;
}

f8_status f8_grad_norm(const f8_tensor* list, int64_t count, f8_norm kind, float* norm, double* sum, void* workspace, size_t workspace_bytes_, void* stream)
{
    if ((int)kind != F8_NORM_2 && (int)kind != F8_NORM_MAX) return F8_ERR_ENUM;
    const f8_status s = check_list(list, count);
    if (s != F8_OK) return s;
    if (!norm && !sum) return F8_ERR_NULL;
    if (!aligned16(workspace) || ((uintptr_t)norm & 3) || ((uintptr_t)sum & 7)) return F8_ERR_ALIGN;
    if (!workspace || workspace_bytes_ < norm_bytes(list, count)) return F8_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    double* const part = (double*)workspace;
    int64_t parts = 0;
    const bool max = kind == F8_NORM_MAX, once = list_bytes(list, count) >= kOnceBytes;
    const auto launch = [&]<int CAP>(const TensorList<CAP>& l) {
        const unsigned b = grad_blocks(l.first[l.count]);
        const auto kernel = max ? (once ? grad_norm_kernel<true, true, CAP> : grad_norm_kernel<true, false, CAP>)
                                : (once ? grad_norm_kernel<false, true, CAP> : grad_norm_kernel<false, false, CAP>);
        kernel<<<b, kGradThreads, 0, st>>>(l, part + parts);
        parts += b;
    };
    if (count <= kFewTensors) for_launches<kFewTensors>(list, nullptr, count, launch);  // (less for the host to copy)
    else for_launches<kTensors>(list, nullptr, count, launch);
    (max ? grad_norm_final_kernel<true> : grad_norm_final_kernel<false>)<<<1, 1024, 0, st>>>(part, parts, norm, sum);
    return last_launch_status();
}

f8_status f8_grad_clip(const f8_tensor* in, const f8_tensor* out, int64_t count, const float* norm, float most, void* stream)
{
    if (!out) out = in;
    f8_status s = check_list(in, count);
    if (s != F8_OK || (s = check_list(out, count)) != F8_OK) return s;
    if (!norm) return F8_ERR_NULL;
    if ((uintptr_t)norm & 3) return F8_ERR_ALIGN;
    if (!(most >= 0.0f)) return F8_ERR_SHAPE;
    for (int64_t i = 0; i < count; ++i) {
        if (in[i].type != out[i].type) return F8_ERR_ENUM;
        const int64_t bytes = in[i].n * element_bytes(in[i]);
        if (in[i].n != out[i].n || (in[i].data != out[i].data && bytes && !apart({in[i].data, bytes}, {out[i].data, bytes}))) return F8_ERR_SHAPE;
    }
    const bool once = list_bytes(in, count) >= kOnceBytes;
    const auto launch = [&]<int CAP>(const TensorList<CAP>& l) {
        const uint32_t steps = l.first[l.count], blocks = kClipBlocks;
        (once ? grad_clip_kernel<true, CAP> : grad_clip_kernel<false, CAP>)<<<steps < blocks ? steps : blocks, kGradThreads, 0, (hipStream_t)stream>>>(l, norm, most);
    };
    if (count <= kFewTensors) for_launches<kFewTensors>(in, out, count, launch);
    else for_launches<kTensors>(in, out, count, launch);
    return last_launch_status();
}

}  // extern "C"
