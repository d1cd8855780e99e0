// The global norm of a list of gradients, and their clipping (gear_grad_norm, gear_clip_grads):
//     norm = sqrt(sum g^2),  c = min(1, max_norm / (norm + 1e-6)),  out = c g.
// Two launches: every block leaves the sum of squares of its share of the values, then every block adds up all shares in one
// order, which gives each of them the same c, and scales its own.  No atomics: the same list gives the same bits.
// Bound by memory: a list that does not fit the L2 is read twice and written once (94 million values in 150 tensors, fp32 and bf16: 171 us for
// 950 MB; blocks of 592 or 1184, four or eight loads ahead, eviction hints, shorter steps backwards are within 3 % of each other, forwards 174).  The second launch walks a block's share
// backwards, so that it begins with what the first one has left in the L2.
// Squares are formed and added in 64 bits: a gradient of 1e-30 or 1e30 has a norm too, and a sum of a billion terms keeps its digits.
#include "common.cuh"
#include "internal.h"

namespace gear {

constexpr int CLIP_THREADS = 256;
constexpr int CLIP_BLOCKS = 1184;          // eight for every SM of a B200: also the shares in the workspace
constexpr int CLIP_SMALL = 32, CLIP_MIDDLE = 256, CLIP_LARGE = 1024;      // tensors a launch can take, as kernel parameters (30 KB of them cost the host 5 us)
constexpr uint32_t CLIP_BACK = 8;          // tiles of a step backwards
static_assert(CLIP_BLOCKS * sizeof(double) <= GEAR_CLIP_WORKSPACE_BYTES, "workspace");

// A tensor's values in vectors of 16 bytes, `head` single values in front of the first.  A tile is `tile` vectors; a
// block goes through neighbouring tiles of a tensor as one stretch.  The single values at both ends belong to the tensor's first tile.
template <int MAX> struct ClipList {
    const void* g[MAX];
    void* out[MAX];
    int64_t n[MAX];
    uint32_t first[MAX + 1];               // tile number of every tensor's first tile
    uint8_t bf16[MAX], head[MAX];
    int count, tile;
};
static_assert(sizeof(ClipList<CLIP_LARGE>) + 256 < 32764, "kernel parameters");

template <bool BF16> struct ClipVec;
template <> struct ClipVec<false> {
    typedef float T;
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 scaled(const uint4& v, float c) {
        float f[4];
        get(v, f);
        return make_uint4(__float_as_uint(f[0] * c), __float_as_uint(f[1] * c), __float_as_uint(f[2] * c), __float_as_uint(f[3] * c));
    }
    static __device__ __forceinline__ float one(float v) { return v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
template <> struct ClipVec<true> {
    typedef __nv_bfloat16 T;
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint4 scaled(const uint4& v, float c) {
        float f[8];
        get(v, f);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i] * c, f[2 * i + 1] * c);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float one(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 round(float v) { return __float2bfloat16(v); }
};

__device__ __forceinline__ double sum_over_block(double v, double* scratch) {      // scratch: one per warp; all threads get the sum
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) scratch[warp] = v;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < CLIP_THREADS / 32; ++w) t += scratch[w];
    return t;
}

// The single values of a tensor: `head` in front of the vectors, the rest behind them.
template <bool BF16, typename Fn> __device__ __forceinline__ void clip_ends(int64_t n, int head, Fn&& fn) {
    constexpr int N = ClipVec<BF16>::N;
    const int64_t nv = (n - head) / N, behind = head + nv * N;
    if ((int)threadIdx.x < head) fn((int64_t)threadIdx.x);
    if (behind + threadIdx.x < n) fn(behind + threadIdx.x);      // fewer than N
}

template <bool BF16> __device__ __forceinline__ double clip_sum_stretch(const void* g, int64_t n, int head, int64_t v0, int64_t vectors) {
    typedef ClipVec<BF16> V;
    const typename V::T* p = static_cast<const typename V::T*>(g);
    const uint4* vec = reinterpret_cast<const uint4*>(p + head);
    const int64_t v1 = min(v0 + vectors, (n - head) / V::N);
    double sum = 0.0;
    int64_t v = v0 + threadIdx.x;
    auto add = [&](const uint4& q) {
        float f[V::N];
        V::get(q, f);
#pragma unroll
        for (int i = 0; i < V::N; ++i) sum = fma((double)f[i], (double)f[i], sum);
    };
    for (; v + 3 * CLIP_THREADS < v1; v += 4 * CLIP_THREADS) {       // four on their way at a time
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = __ldg(vec + v + u * CLIP_THREADS);
#pragma unroll
        for (int u = 0; u < 4; ++u) add(q[u]);
    }
    for (; v < v1; v += CLIP_THREADS) add(__ldg(vec + v));
    if (v0 == 0) clip_ends<BF16>(n, head, [&](int64_t i) { const double f = V::one(p[i]); sum = fma(f, f, sum); });
    return sum;
}

template <bool BF16> __device__ __forceinline__ void clip_scale_stretch(const void* g, void* out, int64_t n, int head, int64_t v0, int64_t vectors, float c) {
    typedef ClipVec<BF16> V;
    typedef typename V::T T;
    const T* p = static_cast<const T*>(g);
    T* o = static_cast<T*>(out);
    const uint4* vec = reinterpret_cast<const uint4*>(p + head);
    const int64_t v1 = min(v0 + vectors, (n - head) / V::N);
    const bool whole = (reinterpret_cast<uintptr_t>(o + head) & 15u) == 0;
    auto put = [&](int64_t v, const uint4& q) {
        const uint4 r = V::scaled(q, c);
        if (whole) reinterpret_cast<uint4*>(o + head)[v] = r;
        else {                                              // out is aligned in another way than grad
            const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
            for (int i = 0; i < V::N; ++i) o[head + v * V::N + i] = e[i];
        }
    };
    int64_t v = v0 + threadIdx.x;
    for (; v + 3 * CLIP_THREADS < v1; v += 4 * CLIP_THREADS) {
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = vec[v + u * CLIP_THREADS];
#pragma unroll
        for (int u = 0; u < 4; ++u) put(v + u * CLIP_THREADS, q[u]);
    }
    for (; v < v1; v += CLIP_THREADS) put(v, vec[v]);
    if (v0 == 0) clip_ends<BF16>(n, head, [&](int64_t i) { o[i] = V::round(V::one(p[i]) * c); });
}

// the tensor a tile belongs to
template <int MAX> __device__ __forceinline__ int clip_tensor_of(const ClipList<MAX>& l, uint32_t t) {
    int lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// a block's share of the tiles
__device__ __forceinline__ void clip_share(uint32_t tiles, uint32_t& t0, uint32_t& t1) {
    t0 = (uint32_t)((uint64_t)tiles * blockIdx.x / gridDim.x);
    t1 = (uint32_t)((uint64_t)tiles * (blockIdx.x + 1) / gridDim.x);
}

// share[b] (+)= sum of squares of block b's tiles; more: the list's tensors follow those of an earlier launch
template <int MAX>
__global__ void __launch_bounds__(CLIP_THREADS)
clip_sum_kernel(const __grid_constant__ ClipList<MAX> l, double* __restrict__ share, int more) {
    __shared__ double scratch[CLIP_THREADS / 32];
    wait_for_predecessor();
    uint32_t t, t1;
    clip_share(l.first[l.count], t, t1);
    double sum = 0.0;
    if (t < t1) {
        int i = clip_tensor_of(l, t);
        for (uint32_t end; t < t1; t = end, ++i) {
            end = min(t1, l.first[i + 1]);
            const int64_t v0 = (int64_t)(t - l.first[i]) * l.tile, vectors = (int64_t)(end - t) * l.tile;
            sum += l.bf16[i] ? clip_sum_stretch<true>(l.g[i], l.n[i], l.head[i], v0, vectors) : clip_sum_stretch<false>(l.g[i], l.n[i], l.head[i], v0, vectors);
        }
    }
    sum = sum_over_block(sum, scratch);
    if (threadIdx.x == 0) share[blockIdx.x] = more ? share[blockIdx.x] + sum : sum;
}

// The shares of all blocks, added up in one order by whoever asks; norm and c from them.
__device__ __forceinline__ double clip_norm(const double* share, int shares, double* scratch) {
    double sum = 0.0;
    for (int b = threadIdx.x; b < shares; b += CLIP_THREADS) sum += __ldcg(share + b);
    return sqrt(sum_over_block(sum, scratch));
}

__global__ void __launch_bounds__(CLIP_THREADS)
clip_norm_kernel(const double* __restrict__ share, int shares, float* __restrict__ norm) {
    __shared__ double scratch[CLIP_THREADS / 32];
    wait_for_predecessor();
    const double r = clip_norm(share, shares, scratch);
    if (threadIdx.x == 0) norm[0] = (float)r;
}

template <int MAX>
__global__ void __launch_bounds__(CLIP_THREADS)
clip_scale_kernel(const __grid_constant__ ClipList<MAX> l, const double* __restrict__ share, int shares, float max_norm, float* __restrict__ norm) {
    __shared__ double scratch[CLIP_THREADS / 32];
    wait_for_predecessor();
    const double r = clip_norm(share, shares, scratch), q = (double)max_norm / (r + 1e-6);
    const float c = q >= 1.0 ? 1.f : (float)q;             // (a NaN stays one)
    if (blockIdx.x == 0 && threadIdx.x == 0) { norm[0] = (float)r; norm[1] = c; }
    uint32_t t0, t1;
    clip_share(l.first[l.count], t0, t1);
    if (t0 >= t1) return;
    int i = clip_tensor_of(l, t1 - 1);
    for (uint32_t t = t1; t > t0;) {                       // backwards, a few tiles at a time
        while (t <= l.first[i]) --i;
        const uint32_t end = t;
        t = max(max(t0, l.first[i]), end > CLIP_BACK ? end - CLIP_BACK : 0u);
        if (c == 1.f && l.out[i] == l.g[i]) continue;
        const int64_t v0 = (int64_t)(t - l.first[i]) * l.tile, vectors = (int64_t)(end - t) * l.tile;
        if (l.bf16[i]) clip_scale_stretch<true>(l.g[i], l.out[i], l.n[i], l.head[i], v0, vectors, c);
        else clip_scale_stretch<false>(l.g[i], l.out[i], l.n[i], l.head[i], v0, vectors, c);
    }
}

// Tensors at .. of a list, as many as a launch takes; `at` moves behind them.  Empty tensors are left out.
template <int MAX> static void clip_fill(ClipList<MAX>& l, const gear_grad* g, int32_t count, int32_t* at, int tile) {
    l.count = 0; l.tile = tile; l.first[0] = 0;
    for (; *at < count && l.count < MAX; ++*at) {
        const gear_grad& t = g[*at];
        if (t.n == 0) continue;
        const int size = t.dtype == GEAR_BF16 ? 2 : 4, i = l.count;
        const int64_t head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(t.grad) & 15u)) & 15u) / size;
        l.g[i] = t.grad; l.out[i] = t.out; l.n[i] = t.n; l.bf16[i] = t.dtype == GEAR_BF16;
        l.head[i] = (uint8_t)(head < t.n ? head : t.n);
        const int64_t tiles = ceil_div((t.n - l.head[i]) / (16 / size), tile);
        l.first[i + 1] = l.first[i] + (uint32_t)(tiles > 1 ? tiles : 1);
        ++l.count;
    }
}

// Tiles of a vector for every thread of a block; longer ones where a launch would count past 2^30 of them.
static int clip_tile(const gear_grad* g, int32_t count) {
    int64_t vectors = 0;
    for (int32_t i = 0; i < count; ++i) vectors += ceil_div(g[i].n, g[i].dtype == GEAR_BF16 ? 8 : 4);
    int64_t tile = CLIP_THREADS;
    while (vectors / tile > (1 << 30)) tile <<= 1;
    return (int)tile;
}

template <int MAX>
static cudaError_t clip_run(const gear_grad* g, int32_t count, bool clip, float max_norm, float* norm, double* share, cudaStream_t st) {
    const int tile = clip_tile(g, count);
    ClipList<MAX> l;
    // all launches over the list have one grid: every share is written
    int64_t tiles = 0;
    for (int32_t i = 0; i < count; ++i) tiles += ceil_div(ceil_div(g[i].n, g[i].dtype == GEAR_BF16 ? 8 : 4), tile);
    const int blocks = (int)(tiles < 1 ? 1 : tiles < CLIP_BLOCKS ? tiles : CLIP_BLOCKS);
    cudaError_t e = cudaSuccess;
    int32_t at = 0, last = 0;
    bool more = false;
    do {
        last = at;
        clip_fill(l, g, count, &at, tile);
        e = launch_now(clip_sum_kernel<MAX>, dim3(blocks), dim3(CLIP_THREADS), 0, st, l, share, (int)more);
        more = true;
    } while (e == cudaSuccess && at < count);
    if (e != cudaSuccess) return e;
    if (!clip) return launch_now(clip_norm_kernel, dim3(1), dim3(CLIP_THREADS), 0, st, static_cast<const double*>(share), blocks, norm);
    // the tensors that were read last come first
    bool single = last == 0;
    e = launch_now(clip_scale_kernel<MAX>, dim3(blocks), dim3(CLIP_THREADS), 0, st, l, static_cast<const double*>(share), blocks, max_norm, norm);
    for (at = 0; !single && at < last && e == cudaSuccess;) {
        clip_fill(l, g, last, &at, tile);
        e = launch_now(clip_scale_kernel<MAX>, dim3(blocks), dim3(CLIP_THREADS), 0, st, l, static_cast<const double*>(share), blocks, max_norm, norm);
    }
    return e;
}

cudaError_t launch_clip(const gear_grad* g, int32_t count, bool clip, float max_norm, float* norm, void* workspace, cudaStream_t st) {
    double* share = static_cast<double*>(workspace);
    return count <= CLIP_SMALL    ? clip_run<CLIP_SMALL>(g, count, clip, max_norm, norm, share, st)
           : count <= CLIP_MIDDLE ? clip_run<CLIP_MIDDLE>(g, count, clip, max_norm, norm, share, st)
                                  : clip_run<CLIP_LARGE>(g, count, clip, max_norm, norm, share, st);
}

}  // namespace gear
