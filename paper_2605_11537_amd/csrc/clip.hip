// The norm over all gradients and their clipping by it: out = g min(1, max_norm / norm), norm = sqrt(sum over all tensors of g^2).
//
// Two launches for up to 96 tensors (their addresses and sizes are the launch's arguments, so that a captured call needs no table in memory).  The
// first gives every workgroup chunks of 16 KB in turn and leaves its sum of squares, in binary64: no square overflows or vanishes, and sums of binary32
// over a billion values would lose digits.  In the second every workgroup adds those sums, in the same order, and scales its chunks.
//
// Bound by memory: 4 or 2 bytes an element are read twice and written once.  The second launch walks the chunks from the last to the first, so that what
// the first has read last is still in the 256 MB cache beside the memory.  1.29 GB of bfloat16: 193 and 469 us (6.7 TB/s read, 5.5 read and written); 8 MB of
// binary32: 4.4 and 5.5 us, a launch and a round trip to memory each, the second with the sum over the first's workgroups.
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

constexpr int CLIP_TENSORS = 96;               // of a launch
constexpr int CLIP_THREADS = 256, CLIP_AHEAD = 4;
constexpr int CLIP_CHUNK = CLIP_THREADS * CLIP_AHEAD * 16;
constexpr int CLIP_KEPT = 12288;               // chunks that the second launch begins with and may find in the cache beside the memory: 192 MB
constexpr int CLIP_BLOCKS = 2048;              // most of a launch: eight to a compute unit
constexpr int CLIP_MAX_TENSORS = 4096;

typedef unsigned clip_u32x4 __attribute__((ext_vector_type(4)));

struct ClipBatch {
    const void *from[CLIP_TENSORS];
    void *to[CLIP_TENSORS];
    long long bytes[CLIP_TENSORS];
    int chunk[CLIP_TENSORS + 1];               // first chunk of a tensor
    unsigned is_bf16[CLIP_TENSORS / 32], loose[CLIP_TENSORS / 32];     // loose: not on 16 bytes
    int n;
};
static_assert(sizeof(ClipBatch) < 3500, "the arguments of a launch");

__device__ __forceinline__ int clip_tensor_of(const ClipBatch &b, int chunk)
{
    int i = 0, past = b.n;
    while (past - i > 1) {
        const int mid = (i + past) >> 1;
        if (b.chunk[mid] <= chunk) i = mid;
        else past = mid;
    }
    return i;
}

__device__ __forceinline__ double square(double s, float v)
{
    const double d = v;
    return fma(d, d, s);
}
template <bool BF16>
__device__ __forceinline__ double squares(double s, clip_u32x4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) s = square(square(s, __uint_as_float(v[i] << 16)), __uint_as_float(v[i] & 0xffff0000u));
        else s = square(s, __uint_as_float(v[i]));
    }
    return s;
}
// max_norm / norm = by 2^-down.  A quotient near or below the smallest normal number would have lost bits, and the gradients that it brings back into the range
// with them; by and its products stay inside.
struct ClipFactor {
    float by;
    int down;
    __device__ __forceinline__ ClipFactor(double f)
    {
        down = f >= 0x1p-100 ? 0 : f >= 0x1p-150 ? 64 : 128;
        by = (float)(down == 0 ? f : f * (down == 64 ? 0x1p64 : 0x1p128));
    }
    __device__ __forceinline__ bool one() const { return by == 1.f; }
    __device__ __forceinline__ float of(float v) const { return __builtin_ldexpf(v * by, -down); }
};
template <bool BF16>
__device__ __forceinline__ clip_u32x4 scaled(clip_u32x4 v, ClipFactor f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) v[i] = pack_bf16x2(f.of(__uint_as_float(v[i] << 16)), f.of(__uint_as_float(v[i] & 0xffff0000u)));
        else v[i] = __float_as_uint(f.of(__uint_as_float(v[i])));
    }
    return v;
}

// f(piece index) for the chunk's whole pieces of 16 bytes, then the elements behind them (all of them, where the tensor is loose)
template <class Whole, class Single>
__device__ __forceinline__ void clip_walk(long long left, bool loose, int size, Whole &&whole, Single &&single)
{
    const int bytes = left < CLIP_CHUNK ? (int)left : CLIP_CHUNK, pieces = loose ? 0 : bytes / 16;
    whole(pieces);
    for (int i = pieces * 16 / size + threadIdx.x; i < bytes / size; i += CLIP_THREADS) single(i);
}

// PASSING: past the caches
template <bool BF16, bool PASSING>
__device__ __forceinline__ double clip_chunk_squares(double s, const char *at, long long left, bool loose)
{
    clip_walk(
        left, loose, BF16 ? 2 : 4,
        [&](int pieces) {
            clip_u32x4 v[CLIP_AHEAD];
#pragma unroll
            for (int i = 0; i < CLIP_AHEAD; ++i) {
                const int p = i * CLIP_THREADS + threadIdx.x;
                v[i] = clip_u32x4{0, 0, 0, 0};
                const clip_u32x4 *q = reinterpret_cast<const clip_u32x4 *>(at + p * 16);
                if (p < pieces) v[i] = PASSING ? __builtin_nontemporal_load(q) : *q;
            }
#pragma unroll
            for (int i = 0; i < CLIP_AHEAD; ++i) s = squares<BF16>(s, v[i]);
        },
        [&](int i) { s = square(s, BF16 ? bf16_to_f32(((const bf16_t *)at)[i]) : ((const float *)at)[i]); });
    return s;
}

__device__ __forceinline__ double clip_sum(double v)
{
    __shared__ double waves[CLIP_THREADS / WAVE];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = waves[0];
#pragma unroll
    for (int w = 1; w < CLIP_THREADS / WAVE; ++w) v += waves[w];
    return v;
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_squares_kernel(ClipBatch b, double *parts)
{
    double s = 0.;
    const int chunks = b.chunk[b.n];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = clip_tensor_of(b, c);
        const long long first = (long long)(c - b.chunk[i]) * CLIP_CHUNK;
        const char *at = (const char *)b.from[i] + first;
        const bool loose = b.loose[i / 32] >> (i % 32) & 1;
        const bool bf16 = b.is_bf16[i / 32] >> (i % 32) & 1, passing = c < chunks - CLIP_KEPT;
        if (bf16 && passing) s = clip_chunk_squares<true, true>(s, at, b.bytes[i] - first, loose);
        else if (bf16) s = clip_chunk_squares<true, false>(s, at, b.bytes[i] - first, loose);
        else if (passing) s = clip_chunk_squares<false, true>(s, at, b.bytes[i] - first, loose);
        else s = clip_chunk_squares<false, false>(s, at, b.bytes[i] - first, loose);
    }
    s = clip_sum(s);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

template <bool BF16>
__device__ __forceinline__ void clip_chunk_scaled(const char *at, char *to, long long left, bool loose, ClipFactor f)
{
    clip_walk(
        left, loose, BF16 ? 2 : 4,
        [&](int pieces) {
            clip_u32x4 v[CLIP_AHEAD];
#pragma unroll
            for (int i = 0; i < CLIP_AHEAD; ++i) {
                const int p = i * CLIP_THREADS + threadIdx.x;
                if (p < pieces) v[i] = *reinterpret_cast<const clip_u32x4 *>(at + p * 16);
            }
#pragma unroll
            for (int i = 0; i < CLIP_AHEAD; ++i) {
                const int p = i * CLIP_THREADS + threadIdx.x;
                // by 1: bit for bit
                if (p < pieces) __builtin_nontemporal_store(f.one() ? v[i] : scaled<BF16>(v[i], f), reinterpret_cast<clip_u32x4 *>(to + p * 16));
            }
        },
        [&](int i) {
            if (BF16) ((bf16_t *)to)[i] = f.one() ? ((const bf16_t *)at)[i] : f32_to_bf16(f.of(bf16_to_f32(((const bf16_t *)at)[i])));
            else ((unsigned *)to)[i] = f.one() ? ((const unsigned *)at)[i] : __float_as_uint(f.of(((const float *)at)[i]));
        });
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_scale_kernel(ClipBatch b, const double *parts, int n_parts, float max_norm, float *norm)
{
    double s = 0.;
    for (int i = threadIdx.x; i < n_parts; i += CLIP_THREADS) s += parts[i];
    const double all = sqrt(clip_sum(s));
    const float reported = (float)all;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = reported;
    // a norm that is no finite number as the caller reads it scales nothing
    const ClipFactor f(all > (double)max_norm && reported < __builtin_inff() ? (double)max_norm / all : 1.);
    const int chunks = b.chunk[b.n];
    for (int c = chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const int i = clip_tensor_of(b, c);
        if (f.one() && b.from[i] == b.to[i]) continue;
        const long long first = (long long)(c - b.chunk[i]) * CLIP_CHUNK;
        const char *at = (const char *)b.from[i] + first;
        char *to = (char *)b.to[i] + first;
        const bool loose = b.loose[i / 32] >> (i % 32) & 1;
        if (b.is_bf16[i / 32] >> (i % 32) & 1) clip_chunk_scaled<true>(at, to, b.bytes[i] - first, loose, f);
        else clip_chunk_scaled<false>(at, to, b.bytes[i] - first, loose, f);
    }
}

int clip_batches(int n) { return n < 1 ? 1 : (n + CLIP_TENSORS - 1) / CLIP_TENSORS; }

// the non-empty tensors from `next` on
bool clip_fill(ClipBatch &b, int &next, const void *const *from, void *const *to, const long long *counts, const int *dtypes, int n)
{
    b = ClipBatch();
    long long chunks = 0;
    for (; next < n && b.n < CLIP_TENSORS; ++next) {
        if (counts[next] == 0) continue;
        const int i = b.n, size = dtypes[next] == MOE_BF16 ? 2 : 4;
        const long long bytes = counts[next] * size, more = (bytes + CLIP_CHUNK - 1) / CLIP_CHUNK;
        if (chunks + more > 0x7fffffff - CLIP_BLOCKS) {
            if (i == 0) return false;          // one tensor of 32 TB
            break;
        }
        b.from[i] = from[next];
        b.to[i] = to[next];
        b.bytes[i] = bytes;
        b.chunk[i] = (int)chunks;
        if (size == 2) b.is_bf16[i / 32] |= 1u << (i % 32);
        if (!aligned16(from[next]) || !aligned16(to[next])) b.loose[i / 32] |= 1u << (i % 32);
        chunks += more;
        b.chunk[++b.n] = (int)chunks;
    }
    return true;
}

struct ClipRange {
    uintptr_t begin, end;
    bool written;
};

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_clip_gradients_workspace_bytes(int n) { return (size_t)clip_batches(n) * CLIP_BLOCKS * sizeof(double); }

extern "C" int moe_clip_gradients(const void *const *gradients, void *const *out, const long long *counts, const int *dtypes, int n, float max_norm,
                                  float *norm, void *ws, size_t ws_bytes, void *stream)
{
    MOE_REQUIRE(n >= 0, MOE_ERR_INVALID_ARG, "moe_clip_gradients: n=%d", n);
    MOE_REQUIRE(n <= CLIP_MAX_TENSORS, MOE_ERR_UNSUPPORTED, "moe_clip_gradients: n=%d > %d", n, CLIP_MAX_TENSORS);
    MOE_REQUIRE(max_norm > 0.f, MOE_ERR_INVALID_ARG, "moe_clip_gradients: max_norm=%g must be above 0", (double)max_norm);
    MOE_REQUIRE(norm && (uintptr_t)norm % 4 == 0 && (n == 0 || (gradients && out && counts && dtypes)), MOE_ERR_INVALID_ARG, "moe_clip_gradients: null or misaligned pointer");
    const size_t need = moe_clip_gradients_workspace_bytes(n);
    MOE_REQUIRE(ws && ws_bytes >= need && aligned16(ws), MOE_ERR_WORKSPACE, "moe_clip_gradients: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    // what is written lies apart from everything else; a gradient may be its own output
    static thread_local ClipRange ranges[2 * CLIP_MAX_TENSORS + 2];
    int m = 0;
    ranges[m++] = {(uintptr_t)norm, (uintptr_t)norm + 4, true};
    ranges[m++] = {(uintptr_t)ws, (uintptr_t)ws + need, true};
    for (int i = 0; i < n; ++i) {
        MOE_REQUIRE(dtypes[i] == MOE_F32 || dtypes[i] == MOE_BF16, MOE_ERR_INVALID_ARG, "moe_clip_gradients: unknown dtype %d", dtypes[i]);
        MOE_REQUIRE(counts[i] >= 0 && counts[i] < 1ll << 45, MOE_ERR_INVALID_ARG, "moe_clip_gradients: a tensor of %lld elements", counts[i]);
        if (counts[i] == 0) continue;
        MOE_REQUIRE(gradients[i] && out[i], MOE_ERR_INVALID_ARG, "moe_clip_gradients: null pointer");
        const int size = dtypes[i] == MOE_BF16 ? 2 : 4;
        const uintptr_t from = (uintptr_t)gradients[i], to = (uintptr_t)out[i], bytes = (uintptr_t)counts[i] * size;
        MOE_REQUIRE(from % size == 0 && to % size == 0, MOE_ERR_INVALID_ARG, "moe_clip_gradients: tensor misaligned");
        ranges[m++] = {to, to + bytes, true};
        if (from != to) ranges[m++] = {from, from + bytes, false};
    }
    std::sort(ranges, ranges + m, [](const ClipRange &a, const ClipRange &b) { return a.begin < b.begin; });
    uintptr_t end = 0, written = 0;
    for (int i = 0; i < m; ++i) {
        MOE_REQUIRE(ranges[i].begin >= (ranges[i].written ? end : written), MOE_ERR_INVALID_ARG,
                    "moe_clip_gradients: an output, norm or the workspace overlaps another tensor, or one is named twice");
        if (ranges[i].end > end) end = ranges[i].end;
        if (ranges[i].written && ranges[i].end > written) written = ranges[i].end;
    }
    hipStream_t st = (hipStream_t)stream;
    double *parts = (double *)ws;
    int n_parts = 0, next = 0;
    ClipBatch b;
    do {
        MOE_REQUIRE(clip_fill(b, next, gradients, out, counts, dtypes, n), MOE_ERR_UNSUPPORTED, "moe_clip_gradients: tensor too large");
        const int blocks = b.chunk[b.n] < CLIP_BLOCKS ? b.chunk[b.n] : CLIP_BLOCKS;
        if (blocks) hipLaunchKernelGGL(clip_squares_kernel, dim3(blocks), dim3(CLIP_THREADS), 0, st, b, parts + n_parts);
        n_parts += blocks;
    } while (next < n);
    next = 0;
    bool first = true;
    do {
        // where one batch holds all tensors it is still there
        if (!first || n > CLIP_TENSORS) clip_fill(b, next, gradients, out, counts, dtypes, n);
        else next = n;
        const int blocks = b.chunk[b.n] < CLIP_BLOCKS ? b.chunk[b.n] : CLIP_BLOCKS;
        if (blocks || first)
            hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks ? blocks : 1), dim3(CLIP_THREADS), 0, st, b, parts, n_parts, max_norm,
                               first ? norm : nullptr);
        first = false;
    } while (next < n);
    MOE_CHECK_LAUNCH("moe_clip_gradients");
    return MOE_OK;
}
