// Common 2-norm of many tensors, and the tensors scaled down where it is above a limit.
//
// norm = sqrt(sum over all tensors and entries of g^2); factor = 1 where max_norm >= norm + eps, else max_norm / (norm + eps) (NaN for a NaN norm),
// formed in 64 bits and rounded to 32 (left in 64 where it would be subnormal); o = rn(g factor).
//
// Tensors are cut into chunks of 32 and 16 KB, dealt out in turn to the blocks of one launch for up to 512 tensors, which it gets as a kernel parameter
// (nothing to copy first; captured by value).  First launch: every thread sums squares of 8 entries in 32 bits and these sums in 64 bits, every block
// leaves one number.  These are added up, in the same order, by every block of the second launch (few chunks) or by one block in between (many).  Second
// launch: every block scales a chunk, last chunk first: those are still in the on-chip cache where all of them do not fit.
#include "layer_ops.cuh"

namespace gemm2m {

namespace {

constexpr int kReadBytes = 32768, kWriteBytes = 16384;      // chunks of the first and of the second launch
constexpr int kClipThreads = 256, kBlocks = 4 * kSms, kFew = 64, kMany = 512;

struct Entry {
    const void* g; void* o;
    int64_t size, ldg, ldo;
    int32_t cols;                         // of a row, 0 where all entries are contiguous
    uint32_t first_read, first_write;     // numbers of its first chunks
    int16_t type, vec;                    // vec: groups of 8 entries are aligned, in g and in o
};
template <int N> struct Table { Entry t[N]; int32_t count; uint32_t read, write; };      // numbers of chunks

__device__ __forceinline__ int64_t place(const Entry& e, int64_t i, int64_t ld) {
    if (!e.cols) return i;
    const int64_t row = i / e.cols;
    return row * ld + (i - row * e.cols);
}

// Sum of the squares of eight entries.  In 32 bits where neither the largest can overflow nor what underflows can matter (squares below 2^-126 against a sum of
// 2^-100 or more: less than its rounding); otherwise, and for sums that are not finite, in 64 bits.
__device__ __forceinline__ double squares8(const float (&v)[8]) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j] * v[j];
    if (s >= 0x1p-100f && s <= 0x1p126f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) d += (double)v[j] * (double)v[j];
    return d;
}

__device__ __forceinline__ double block_sum(double v, double* warps) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) v += warps[w];
    return v;
}

// The entry that chunk c belongs to.
template <bool READ, int N>
__device__ __forceinline__ int entry_of(const Table<N>& t, uint32_t c) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((READ ? t.t[mid].first_read : t.t[mid].first_write) <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The groups of eight entries of chunk c of a tensor that a thread deals with.  `meanwhile` runs when the loads are on their way.
template <typename T, int BYTES, typename M, typename F>
__device__ __forceinline__ void for_chunk(const Entry& e, uint32_t c, M&& meanwhile, F&& f) {
    constexpr int kChunk = BYTES / (int)sizeof(T), kGroups = kChunk / (8 * kClipThreads);
    const int64_t base = (int64_t)c * kChunk;
    const T* g = (const T*)e.g;
    if (e.vec && base + kChunk <= e.size) {
        Raw8<T> raw[kGroups];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) raw[k] = load8_rw<T>(g + place(e, base + (k * kClipThreads + threadIdx.x) * 8, e.ldg));
        meanwhile();
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            float v[8];
            to_floats8<T>(raw[k], v);
            f(v, base + (k * kClipThreads + threadIdx.x) * 8, 8);
        }
        return;
    }
    meanwhile();
    // neighbouring threads take neighbouring entries; (no branches around the loads: beyond the end they read the last entry)
#pragma unroll 2
    for (int k = 0; k < kGroups; ++k) {
        if (base + k * 8 * kClipThreads >= e.size) break;
        float v[8];
        T t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = g[place(e, min(base + (k * 8 + j) * kClipThreads + threadIdx.x, e.size - 1), e.ldg)];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = base + (k * 8 + j) * kClipThreads + threadIdx.x < e.size ? to_float<T>(t[j]) : 0.f;
        f(v, base + k * 8 * kClipThreads + threadIdx.x, 0);
    }
}

// Chunks dealt out to four blocks on every SM, a partial sum each.  Bound by memory (705 million f32 entries: 389 us, 7.25 TB/s, some of them still in the on-chip cache; 54 million in bf16,
// 108 MB: 26 us from a cold start.  Rows apart cost a division per group of eight entries, or per entry where they are not aligned: 1.6 GB of f32 as 24 views 236 us, 225 as 8 whole matrices; of 3999
// columns on odd boundaries 919).
template <int N>
__global__ void __launch_bounds__(kClipThreads, 4) squares_kernel(const __grid_constant__ Table<N> t, double* partials) {
    __shared__ double warps[kClipThreads / 32];
    wait_for_prior_kernels();
    double sum = 0.0;
    auto add = [&](const float (&v)[8], int64_t, int) { sum += squares8(v); };
    int at = entry_of<true>(t, blockIdx.x);
    for (uint32_t c = blockIdx.x; c < t.read; c += gridDim.x) {
        const Entry& e = t.t[at];
        auto meanwhile = [&] { at = entry_of<true>(t, c + gridDim.x); };
        if (e.type == kF32) for_chunk<float, kReadBytes>(e, c - e.first_read, meanwhile, add);
        else if (e.type == kF16) for_chunk<__half, kReadBytes>(e, c - e.first_read, meanwhile, add);
        else for_chunk<__nv_bfloat16, kReadBytes>(e, c - e.first_read, meanwhile, add);
    }
    sum = block_sum(sum, warps);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

// The sum of all partial sums, in an order that goes by their number alone.
__device__ __forceinline__ double total_of(const double* partials, int64_t count, double* warps) {
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += kClipThreads) v += partials[i];
    return block_sum(v, warps);
}

__global__ void __launch_bounds__(kClipThreads) fold_kernel(const double* partials, int64_t count, double* total, float* norm) {
    __shared__ double warps[kClipThreads / 32];
    wait_for_prior_kernels();
    const double sum = total_of(partials, count, warps);
    if (threadIdx.x) return;
    *total = sum;
    if (norm) *norm = (float)sqrt(sum);
}

// Chunk c of a tensor times a factor that 32 bits hold as a subnormal number or not at all: it would lose bits, which results of ordinary size would lose too.  (As a branch around each
// product in the kernel below, or as two factors for all, it costs that kernel registers, and 54 million bf16 entries 13 and 10 % of their time, 705 million f32 entries 2 and 20 %.)
__device__ __noinline__ void scale_far(const Entry& e, uint32_t c, double factor) {
    auto as = [&](auto kind) {
        using T = decltype(kind);
        constexpr int kChunk = kWriteBytes / (int)sizeof(T);
        const int64_t end = min(e.size, (int64_t)(c + 1) * kChunk);
        for (int64_t i = (int64_t)c * kChunk + threadIdx.x; i < end; i += kClipThreads)
            ((T*)e.o)[place(e, i, e.ldo)] = from_float<T>((float)((double)to_float<T>(((const T*)e.g)[place(e, i, e.ldg)]) * factor));
    };
    if (e.type == kF32) as(float());
    else if (e.type == kF16) as(__half());
    else as(__nv_bfloat16());
}

// A block per chunk, which it scales.  (705 million f32 entries: 826 us, 6.8 TB/s; when that was 6.9, 6.4 with chunks of 32 KB and 5.6 with these
// dealt out to four blocks on every SM.  As views of columns on odd boundaries, entry by entry, 2.1 TB/s.)
template <int N>
__global__ void __launch_bounds__(kClipThreads, 6) scale_kernel(const __grid_constant__ Table<N> t, const double* partials, int64_t count, float max_norm, float eps, float* norm) {
    __shared__ double warps[kClipThreads / 32];
    const uint32_t c = t.write - 1 - blockIdx.x;
    const Entry& e = t.t[entry_of<false>(t, c)];
    wait_for_prior_kernels();
    const double size = sqrt(count == 1 ? *partials : total_of(partials, count, warps));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)size;
    const double room = size + (double)eps;
    const float factor = (double)max_norm >= room ? 1.f : (float)((double)max_norm / room);      // (NaN: the second)
    if (factor == 1.f && e.o == e.g) return;
    if (factor < 0x1p-126f) return scale_far(e, c - e.first_write, (double)max_norm / room);
    auto scale = [&](auto kind) {
        using T = decltype(kind);
        for_chunk<T, kWriteBytes>(e, c - e.first_write, [] {}, [&](const float (&v)[8], int64_t from, int whole) {
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) out[j] = v[j] * factor;
            if (whole) {
                store8_as<T>((T*)e.o + place(e, from, e.ldo), out, true, 8);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (from + j * kClipThreads < e.size) ((T*)e.o)[place(e, from + j * kClipThreads, e.ldo)] = from_float<T>(out[j]);
            }
        });
    };
    if (e.type == kF32) scale(float());
    else if (e.type == kF16) scale(__half());
    else scale(__nv_bfloat16());
}

// Up to N tensors as a kernel parameter; returns how many were taken.
template <int N>
int64_t fill(Table<N>* t, const GradTensor* g, int64_t count) {
    t->count = 0;
    t->read = t->write = 0;
    int64_t i = 0;
    for (; i < count && t->count < N; ++i) {
        const int64_t size = g[i].rows * g[i].cols;
        if (size == 0) continue;
        const int es = g[i].type == kF32 ? 4 : 2;
        const bool flat = g[i].rows == 1 || (g[i].ldg == g[i].cols && g[i].ldo == g[i].cols);
        const bool rows_vec = flat || (g[i].cols % 8 == 0 && g[i].ldg * es % 16 == 0 && g[i].ldo * es % 16 == 0);
        const bool vec = rows_vec && (((uintptr_t)g[i].g | (uintptr_t)g[i].o) & 15) == 0;
        t->t[t->count++] = {g[i].g, g[i].o, size, g[i].ldg, g[i].ldo, flat ? 0 : (int32_t)g[i].cols, t->read, t->write, (int16_t)g[i].type, (int16_t)(vec ? 1 : 0)};
        t->read += (uint32_t)((size * es + kReadBytes - 1) / kReadBytes);
        t->write += (uint32_t)((size * es + kWriteBytes - 1) / kWriteBytes);
    }
    return i;
}

int blocks_for(uint32_t chunks) { return chunks < (uint32_t)kBlocks ? (int)chunks : kBlocks; }

template <int N>
cudaError_t launch_all(const GradTensor* g, int64_t count, bool scale, float max_norm, float eps, float* norm, double* partials, cudaStream_t st, int launches[2]) {
    Table<N> t;
    double* total = partials;
    double* part = partials + 1;
    int64_t parts = 0;
    int tables = 0;
    for (int64_t i = 0; i < count; ++tables) {
        i += fill(&t, g + i, count - i);
        if (t.read == 0) continue;
        const int blocks = blocks_for(t.read);
        cudaError_t err = launch_chained(squares_kernel<N>, dim3(blocks), dim3(kClipThreads), 0, st, t, part + parts);
        if (err != cudaSuccess) return err;
        parts += blocks;
        ++launches[0];
    }
    // With few chunks every block of the second launch adds the partial sums up itself; with more of them than of partial sums, with several tables, or no tensor to
    // scale, one block does.
    if (tables != 1 || !scale || parts == 0 || t.write > (uint32_t)kBlocks) {
        cudaError_t err = launch_chained(fold_kernel, dim3(1), dim3(kClipThreads), 0, st, (const double*)part, parts, total, norm);
        if (err != cudaSuccess) return err;
        ++launches[0];
        part = total;
        parts = 1;
        norm = nullptr;
    }
    if (!scale) return cudaSuccess;
    for (int64_t i = 0; i < count;) {
        if (tables != 1) i += fill(&t, g + i, count - i);
        else i = count;
        if (t.read == 0) continue;
        cudaError_t err = launch_chained(scale_kernel<N>, dim3(t.write), dim3(kClipThreads), 0, st, t, (const double*)part, parts, max_norm, eps, norm);
        if (err != cudaSuccess) return err;
        ++launches[1];
    }
    return cudaSuccess;
}

}  // namespace

int64_t clip_partials(int64_t count) { return 1 + (count / kMany + 1) * kBlocks; }

cudaError_t launch_clip_gradients(const GradTensor* t, int64_t count, bool scale, float max_norm, float eps, float* norm, double* partials, cudaStream_t st,
                                  int launches[2]) {
    // a parameter of 4 KB or one of 30 KB, which costs more to launch
    if (count <= kFew) return launch_all<kFew>(t, count, scale, max_norm, eps, norm, partials, st, launches);
    return launch_all<kMany>(t, count, scale, max_norm, eps, norm, partials, st, launches);
}

}  // namespace gemm2m
