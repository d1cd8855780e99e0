// Rows of a normed Dense Part: root-mean-square norm with the residual's addition and an 8-bit (or fp32, bf16) output, its
// gradients, and the 8-bit form of rows and weights (gear_rms_norm, gear_rms_norm_backward, gear_q8_rows, gear_q8_weights).
//
//     y = x + res;  h = y r w,  r = 1 / sqrt(mean y^2 + eps);  per 128 columns: scale = max |h| / 448, q = e4m3(h / scale)
//     dx = r g - y r^3 (sum g y) / cols + dres,  g = dout w;   dw = sum over the rows of dout y r
//
// Bound by memory: every value is read once and written once.  A row stays in the registers of the warps that share it, in the
// type it came in, from its load to its output; a block of 128 columns belongs to one warp (to half a warp where lanes hold 16
// bytes of bf16), so that its largest magnitude needs no shared memory.  Rows wider than the registers go through the kernels
// at the end, which read them again from the L2.
#include "internal.h"
#include "q8.cuh"

namespace gear {

// One lane's part of a chunk of columns that a warp holds.  VEC: E consecutive values in one load; else the lane has every 32nd value
// (any alignment, any width; a warp's loads are still whole lines).
template <typename T, bool VEC> struct Chunk;
template <> struct Chunk<float, true> {
    static constexpr int E = 4, COLS = 128, Q = 128;          // values, columns of the chunk
    float4 v;
    static __device__ __forceinline__ int col(int lane, int e) { return lane * 4 + e; }
    static __device__ __forceinline__ bool in(int lane, int, int left) { return lane * 4 < left; }      // (widths are multiples of E)
    __device__ __forceinline__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p, int lane, int left) { if (lane * 4 < left) v = *reinterpret_cast<const float4*>(p + lane * 4); else zero(); }
    __device__ __forceinline__ void store(float* p, int lane, int left) const { if (lane * 4 < left) *reinterpret_cast<float4*>(p + lane * 4) = v; }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    __device__ __forceinline__ void set(const float (&f)[4]) { v = make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Chunk<__nv_bfloat16, true> {
    static constexpr int E = 8, COLS = 256, Q = 128;
    uint4 v;
    static __device__ __forceinline__ int col(int lane, int e) { return lane * 8 + e; }
    static __device__ __forceinline__ bool in(int lane, int, int left) { return lane * 8 < left; }
    __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int lane, int left) { if (lane * 8 < left) v = *reinterpret_cast<const uint4*>(p + lane * 8); else zero(); }
    __device__ __forceinline__ void store(__nv_bfloat16* p, int lane, int left) const { if (lane * 8 < left) *reinterpret_cast<uint4*>(p + lane * 8) = v; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <typename T> struct Chunk<T, false> {
    static constexpr int E = 4, COLS = 128, Q = 128;
    T v[4];
    static __device__ __forceinline__ int col(int lane, int e) { return lane + 32 * e; }
    static __device__ __forceinline__ bool in(int lane, int e, int left) { return lane + 32 * e < left; }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (T)0.f;
    }
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = lane + 32 * e < left ? p[lane + 32 * e] : (T)0.f;
    }
    __device__ __forceinline__ void store(T* p, int lane, int left) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (lane + 32 * e < left) p[lane + 32 * e] = v[e];
    }
    __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)v[e];
    }
    __device__ __forceinline__ void set(const float (&f)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (T)f[e];
    }
};

// E values of a vector of weights (null: ones)
template <bool VEC, int E> __device__ __forceinline__ void load_weight(const float* w, int lane, int left, float (&f)[E]) {
    if (w == nullptr) {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = 1.f;
    } else if (VEC) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 v = lane * E + e < left ? __ldg(reinterpret_cast<const float4*>(w + lane * E + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
            f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = lane + 32 * e < left ? __ldg(w + lane + 32 * e) : 0.f;
    }
}

// E results of a lane to a row of `dtype`.  For GEAR_E4M3 also the scales of the chunk's blocks, scale[0] the first one's.  The
// whole warp calls.
template <bool VEC, int E> __device__ __forceinline__ void put_row(void* row, int col0, int lane, int left, int dtype, float* scale, const float (&h)[E]) {
    if (dtype == GEAR_E4M3) {
        uint32_t m = 0u;
#pragma unroll
        for (int e = 0; e < E; ++e) m = max(m, q8_magnitude(h[e]));
        constexpr int LANES = VEC && E == 8 ? 16 : 32;                // lanes that share a block
        m = __reduce_max_sync(LANES == 32 ? 0xffffffffu : lane < 16 ? 0xffffu : 0xffff0000u, m);
        float inv;
        const float s = q8_scale(m, inv);
        if (lane % LANES == 0 && (lane / LANES) * Q8_BLOCK < left) scale[lane / LANES] = s;
        uint8_t* q = static_cast<uint8_t*>(row) + col0;
        if (VEC) {
            uint32_t w[E / 4];
#pragma unroll
            for (int e = 0; e < E; e += 4) w[e / 4] = (uint32_t)q8_pair(h[e] * inv, h[e + 1] * inv) | (uint32_t)q8_pair(h[e + 2] * inv, h[e + 3] * inv) << 16;
            if (lane * E < left) {
                if (E == 4) *reinterpret_cast<uint32_t*>(q + lane * 4) = w[0];
                else *reinterpret_cast<uint2*>(q + lane * 8) = make_uint2(w[0], w[E / 4 - 1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (lane + 32 * e < left) q[lane + 32 * e] = q8_one(h[e] * inv);
        }
    } else if (dtype == GEAR_BF16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(row) + col0;
        if (VEC) {
            uint32_t w[E / 2];
#pragma unroll
            for (int e = 0; e < E; e += 2) { const __nv_bfloat162 p = __floats2bfloat162_rn(h[e], h[e + 1]); w[e / 2] = *reinterpret_cast<const uint32_t*>(&p); }
            if (lane * E < left) {
                if (E == 4) *reinterpret_cast<uint2*>(o + lane * 4) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint4*>(o + lane * 8) = make_uint4(w[0], w[1], w[E / 2 - 2], w[E / 2 - 1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (lane + 32 * e < left) o[lane + 32 * e] = __float2bfloat16(h[e]);
        }
    } else {
        float* o = static_cast<float*>(row) + col0;
#pragma unroll
        for (int e = 0; e < E; e += VEC ? 4 : 1) {
            if (VEC) { if (lane * E + e < left) *reinterpret_cast<float4*>(o + lane * E + e) = make_float4(h[e], h[e + (VEC ? 1 : 0)], h[e + (VEC ? 2 : 0)], h[e + (VEC ? 3 : 0)]); }
            else if (lane + 32 * e < left) o[lane + 32 * e] = h[e];
        }
    }
}

__device__ __forceinline__ int64_t live_rows(const NormArgs& a) {
    if (!a.d_n) return a.n;
    const int64_t live = *a.d_n;
    return live < a.n ? (live < 0 ? 0 : live) : a.n;
}
// the row of x that row k reads, or null (an ID outside the table)
template <typename T> __device__ __forceinline__ const T* row_of_x(const NormArgs& a, int64_t k, bool report) {
    if (!a.ids) return static_cast<const T*>(a.x) + k * a.ldx;
    const int64_t id = a.ids[k];
    if (id >= 0 && id < a.vocab) return static_cast<const T*>(a.x) + id * a.ldx;
    if (report && a.status) atomicOr(a.status, GEAR_DEV_BAD_ID);
    return nullptr;
}
template <typename T> __device__ __forceinline__ void* row_of_out(const NormArgs& a, int64_t k) {
    return static_cast<char*>(a.out) + k * a.ld_out * (a.out_dtype == GEAR_E4M3 ? 1 : a.out_dtype == GEAR_BF16 ? 2 : 4);
}

// v summed over the W warps that share a row; scratch: W values of that row.  (All warps of the block call.)
template <int W> __device__ __forceinline__ float sum_over_row(float v, float* scratch, int part) {
    v = warp_sum(v);
    if (W == 1) return v;
    if ((threadIdx.x & 31) == 0) scratch[part] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) t += scratch[w];
    return t;
}

constexpr int NORM_WARPS = 4;                    // warps per block where a warp has a row of its own

// W warps per row (1, or all eight of the block), C chunks per warp: chunk c of the row belongs to warp c % W.
template <typename T, bool VEC, int W, int C>
__global__ void __launch_bounds__(W == 1 ? 32 * NORM_WARPS : 32 * W)
rms_norm_kernel(const NormArgs a) {
    typedef Chunk<T, VEC> Ch;
    constexpr int ROWS = W == 1 ? NORM_WARPS : 1;
    __shared__ float scratch[W];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = W == 1 ? 0 : warp;
    const int64_t k = (int64_t)blockIdx.x * ROWS + (W == 1 ? warp : 0);
    if (k >= live_rows(a)) return;               // (uniform over the warps of a row)
    const T* x = row_of_x<T>(a, k, lane == 0 && part == 0);
    Ch y[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col0 = (c * W + part) * Ch::COLS;
        if (col0 < a.cols && x) y[c].load(x + col0, lane, a.cols - col0); else y[c].zero();
    }
    if (a.res) {
        const T* res = static_cast<const T*>(a.res) + k * a.ld_res;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col0 = (c * W + part) * Ch::COLS;
            if (col0 >= a.cols) continue;
            Ch r;
            r.load(res + col0, lane, a.cols - col0);
            float f[Ch::E], g[Ch::E];
            y[c].get(f); r.get(g);
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) f[e] += g[e];
            y[c].set(f);                         // the residual stream is kept in its own type; the norm is the kept sum's
        }
    }
    float sum = 0.f;
    if (a.normed) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float f[Ch::E];
            y[c].get(f);
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) sum = fmaf(f[e], f[e], sum);
        }
        sum = sum_over_row<W>(sum, scratch, part);
    }
    if (a.res_out) {
        T* o = static_cast<T*>(a.res_out) + k * a.ld_res_out;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col0 = (c * W + part) * Ch::COLS;
            if (col0 < a.cols) y[c].store(o + col0, lane, a.cols - col0);
        }
    }
    const float r = a.normed ? 1.0f / sqrtf(sum / (float)a.cols + a.eps) : 1.f;
    void* out = row_of_out<T>(a, k);
    float* scale = a.scale ? a.scale + k * a.blocks : nullptr;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col0 = (c * W + part) * Ch::COLS;
        if (col0 >= a.cols) continue;
        float f[Ch::E], w[Ch::E];
        y[c].get(f);
        if (a.normed) {
            load_weight<VEC, Ch::E>(a.weight ? a.weight + col0 : nullptr, lane, a.cols - col0, w);
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) f[e] = f[e] * r * w[e];
        }
        put_row<VEC, Ch::E>(out, col0, lane, a.cols - col0, a.out_dtype, scale + col0 / Q8_BLOCK, f);
    }
}

// Rows of any width: eight warps per row, three passes over it.
template <typename T>
__global__ void __launch_bounds__(256)
rms_norm_wide_kernel(const NormArgs a) {
    typedef Chunk<T, false> Ch;
    __shared__ float scratch[8];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t live = live_rows(a);
    for (int64_t k = blockIdx.x; k < live; k += gridDim.x) {
        const T* x = row_of_x<T>(a, k, threadIdx.x == 0);
        const T* res = a.res ? static_cast<const T*>(a.res) + k * a.ld_res : nullptr;
        T* kept = a.res_out ? static_cast<T*>(a.res_out) + k * a.ld_res_out : nullptr;
        // y of a chunk; once it has been kept it is read from there (res_out may be what it was made from)
        auto get = [&](int col0, bool from_kept, float (&f)[Ch::E]) {
            Ch y;
            if (from_kept) { y.load(kept + col0, lane, a.cols - col0); y.get(f); return; }
            if (x) y.load(x + col0, lane, a.cols - col0); else y.zero();
            y.get(f);
            if (res) {
                Ch r;
                float g[Ch::E];
                r.load(res + col0, lane, a.cols - col0); r.get(g);
#pragma unroll
                for (int e = 0; e < Ch::E; ++e) f[e] += g[e];
                y.set(f); y.get(f);
            }
            if (kept) y.store(kept + col0, lane, a.cols - col0);
        };
        float sum = 0.f;
        if (a.normed || kept)
            for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
                float f[Ch::E];
                get(col0, false, f);
#pragma unroll
                for (int e = 0; e < Ch::E; ++e) sum = fmaf(f[e], f[e], sum);
            }
        sum = sum_over_row<8>(sum, scratch, part);
        const float r = a.normed ? 1.0f / sqrtf(sum / (float)a.cols + a.eps) : 1.f;
        void* out = row_of_out<T>(a, k);
        float* scale = a.scale ? a.scale + k * a.blocks : nullptr;
        for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
            float f[Ch::E], w[Ch::E];
            get(col0, kept != nullptr, f);
            if (a.normed) {
                load_weight<false, Ch::E>(a.weight ? a.weight + col0 : nullptr, lane, a.cols - col0, w);
#pragma unroll
                for (int e = 0; e < Ch::E; ++e) f[e] = f[e] * r * w[e];
            }
            put_row<false, Ch::E>(out, col0, lane, a.cols - col0, a.out_dtype, scale + col0 / Q8_BLOCK, f);
        }
        __syncthreads();                         // scratch is free for the next row
    }
}

// ---------------------------------------------------------------- gradients
// Blocks walk the rows (of stripes one grid apart); a lane adds up its columns' part of dw in registers.  At the end the warps of a
// block with a row each add theirs up in shared memory, one after the other, and the block's sums go to its row of `parts`: the
// order is the same in every run.
template <typename T, bool VEC, int W, int C>
__global__ void __launch_bounds__(W == 1 ? 32 * NORM_WARPS : 32 * W)
rms_norm_back_kernel(const NormArgs a) {
    typedef Chunk<T, VEC> Ch;
    constexpr int ROWS = W == 1 ? NORM_WARPS : 1;
    __shared__ float scratch[2][2][W];
    extern __shared__ float dw_sum[];            // W == 1: [cols]
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = W == 1 ? 0 : warp;
    const int64_t live = live_rows(a);
    const float inv_cols = 1.0f / (float)a.cols;
    float dw[C][Ch::E];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < Ch::E; ++e) dw[c][e] = 0.f;
    int odd = 0;
    for (int64_t k = (int64_t)blockIdx.x * ROWS + (W == 1 ? warp : 0); k < live; k += (int64_t)gridDim.x * ROWS, odd ^= 1) {
        const T* x = row_of_x<T>(a, k, lane == 0 && part == 0);
        const T* dout = static_cast<const T*>(a.dout) + k * a.ld_dout;
        Ch y[C], g[C];
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col0 = (c * W + part) * Ch::COLS;
            if (col0 < a.cols) { if (x) y[c].load(x + col0, lane, a.cols - col0); else y[c].zero(); g[c].load(dout + col0, lane, a.cols - col0); }
            else { y[c].zero(); g[c].zero(); }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col0 = (c * W + part) * Ch::COLS;
            if (col0 >= a.cols) continue;
            float f[Ch::E], d[Ch::E], w[Ch::E];
            y[c].get(f); g[c].get(d);
            load_weight<VEC, Ch::E>(a.weight ? a.weight + col0 : nullptr, lane, a.cols - col0, w);
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) { sq = fmaf(f[e], f[e], sq); dot = fmaf(d[e] * w[e], f[e], dot); }
        }
        // (two sets of scratch words in turn: a row's sums are read by all before the row after the next one's are written)
        sq = warp_sum(sq); dot = warp_sum(dot);
        if (W > 1) {
            if (lane == 0) { scratch[odd][0][part] = sq; scratch[odd][1][part] = dot; }
            __syncthreads();
            sq = dot = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) { sq += scratch[odd][0][w]; dot += scratch[odd][1][w]; }
        }
        const float r = 1.0f / sqrtf(sq * inv_cols + a.eps);
        const float q = r * r * (dot * inv_cols);          // dx = r (g - y q): r alone may be large where y is small
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col0 = (c * W + part) * Ch::COLS;
            if (col0 >= a.cols) continue;
            float f[Ch::E], d[Ch::E], w[Ch::E];
            y[c].get(f); g[c].get(d);
            if (a.dx) {
                load_weight<VEC, Ch::E>(a.weight ? a.weight + col0 : nullptr, lane, a.cols - col0, w);
                float o[Ch::E];
#pragma unroll
                for (int e = 0; e < Ch::E; ++e) o[e] = r * (d[e] * w[e] - f[e] * q);
                if (a.dres) {
                    Ch s;
                    float t[Ch::E];
                    s.load(static_cast<const T*>(a.dres) + k * a.ld_dres + col0, lane, a.cols - col0);
                    s.get(t);
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e) o[e] += t[e];
                }
                Ch s;
                s.set(o);
                s.store(static_cast<T*>(a.dx) + k * a.ld_dx + col0, lane, a.cols - col0);
            }
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) dw[c][e] = fmaf(d[e] * r, f[e], dw[c][e]);
        }
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.x * a.cols;
    if (W == 1) {
        for (int turn = 0; turn < ROWS; ++turn) {
            if (warp == turn)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e) {
                        const int col = c * Ch::COLS + Ch::col(lane, e);
                        if (col < a.cols) dw_sum[col] = turn == 0 ? dw[c][e] : dw_sum[col] + dw[c][e];
                    }
            __syncthreads();
        }
        for (int col = threadIdx.x; col < a.cols; col += 32 * NORM_WARPS) to[col] = dw_sum[col];
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < Ch::E; ++e) {
                const int col = (c * W + part) * Ch::COLS + Ch::col(lane, e);
                if (col < a.cols) to[col] = dw[c][e];
            }
    }
}

// Rows of any width: two passes over a row; dw is added up in the block's row of `parts`, which belongs to it alone.
template <typename T>
__global__ void __launch_bounds__(256)
rms_norm_back_wide_kernel(const NormArgs a) {
    typedef Chunk<T, false> Ch;
    __shared__ float scratch[2][8];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t live = live_rows(a);
    float* to = a.parts ? a.parts + (int64_t)blockIdx.x * a.cols : nullptr;
    if (to) {
        for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS)
            for (int e = 0; e < Ch::E; ++e) if (Ch::in(lane, e, a.cols - col0)) to[col0 + Ch::col(lane, e)] = 0.f;
    }
    for (int64_t k = blockIdx.x; k < live; k += gridDim.x) {
        const T* x = row_of_x<T>(a, k, threadIdx.x == 0);
        const T* dout = static_cast<const T*>(a.dout) + k * a.ld_dout;
        float sq = 0.f, dot = 0.f;
        for (int pass = 0; pass < 2; ++pass) {
            const float inv_cols = 1.0f / (float)a.cols;
            const float r = 1.0f / sqrtf(sq * inv_cols + a.eps), q = r * r * (dot * inv_cols);      // (second pass)
            for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
                const int left = a.cols - col0;
                Ch y, g;
                float f[Ch::E], d[Ch::E], w[Ch::E], o[Ch::E];
                if (x) y.load(x + col0, lane, left); else y.zero();
                g.load(dout + col0, lane, left);
                y.get(f); g.get(d);
                load_weight<false, Ch::E>(a.weight ? a.weight + col0 : nullptr, lane, left, w);
                if (pass == 0) {
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e) { sq = fmaf(f[e], f[e], sq); dot = fmaf(d[e] * w[e], f[e], dot); }
                    continue;
                }
                if (a.dx) {
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e) o[e] = r * (d[e] * w[e] - f[e] * q);
                    Ch s;
                    if (a.dres) {
                        float t[Ch::E];
                        s.load(static_cast<const T*>(a.dres) + k * a.ld_dres + col0, lane, left);
                        s.get(t);
#pragma unroll
                        for (int e = 0; e < Ch::E; ++e) o[e] += t[e];
                    }
                    s.set(o);
                    s.store(static_cast<T*>(a.dx) + k * a.ld_dx + col0, lane, left);
                }
                if (to)
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e)
                        if (Ch::in(lane, e, left)) { float* p = to + col0 + Ch::col(lane, e); *p = fmaf(d[e] * r, f[e], *p); }
            }
            if (pass == 0) { sq = sum_over_row<8>(sq, scratch[0], part); dot = sum_over_row<8>(dot, scratch[1], part); }
        }
        __syncthreads();
    }
}

// dw[c] = the blocks' sums added up, always in the same order: 32 columns a block, eight warps over the rows
__global__ void __launch_bounds__(256)
norm_dweight_kernel(const float* __restrict__ parts, int rows, int cols, float* __restrict__ dweight) {
    __shared__ float s[8][33];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float t = 0.f;
    if (col < cols) for (int r = warp; r < rows; r += 8) t += __ldcg(parts + (int64_t)r * cols + col);
    s[warp][lane] = t;
    __syncthreads();
    if (warp == 0 && col < cols) {
        t = 0.f;
        for (int w = 0; w < 8; ++w) t += s[w][lane];
        dweight[col] = t;
    }
}

// ---------------------------------------------------------------- weights
// One block per 128 x 128 weights: the block's values in shared memory (rows of 129 words, so that a warp may walk them in both
// directions), their largest magnitude, both copies written in whole rows of the block.
__global__ void __launch_bounds__(256)
q8_weights_kernel(const float* __restrict__ W, int64_t ldw, int K, int N, uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale,
                  uint8_t* __restrict__ qt, int64_t ldqt, float* __restrict__ scale_t) {
    extern __shared__ float tile[];              // [128][129]
    __shared__ uint32_t most[8];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k0 = blockIdx.x * Q8_BLOCK, n0 = blockIdx.y * Q8_BLOCK, kn = min(Q8_BLOCK, K - k0), nn = min(Q8_BLOCK, N - n0);
    uint32_t m = 0u;
    for (int k = warp; k < kn; k += 8) {
        const float* row = W + (int64_t)(k0 + k) * ldw + n0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = lane + 32 * e;
            if (n >= nn) continue;
            const float v = __ldg(row + n);
            tile[k * 129 + n] = v;
            m = max(m, q8_magnitude(v));
        }
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) most[warp] = m;
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = max(m, most[w]);
    float inv;
    const float s = q8_scale(m, inv);
    if (threadIdx.x == 0) {
        if (q) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
        if (qt) scale_t[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = s;
    }
    if (q)
        for (int n = warp; n < nn; n += 8) {
            uint8_t* row = q + (int64_t)(n0 + n) * ldq + k0;
#pragma unroll
            for (int e = 0; e < 4; ++e) if (lane + 32 * e < kn) row[lane + 32 * e] = q8_one(tile[(lane + 32 * e) * 129 + n] * inv);
        }
    if (qt)
        for (int k = warp; k < kn; k += 8) {
            uint8_t* row = qt + (int64_t)(k0 + k) * ldqt + n0;
#pragma unroll
            for (int e = 0; e < 4; ++e) if (lane + 32 * e < nn) row[lane + 32 * e] = q8_one(tile[k * 129 + lane + 32 * e] * inv);
        }
}

// ---------------------------------------------------------------- host side
static bool on16(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0; }

// whether all rows start on 16-byte boundaries and hold whole vectors (an 8-bit row: on 8-byte boundaries, a lane's piece of it)
static bool vectors(const NormArgs& a, int size) {
    const int64_t vec = 16 / size;
    if (a.cols % vec || !on16(a.x, a.ldx, size) || (a.weight && !on16(a.weight, 0, 4))) return false;
    if ((a.res && !on16(a.res, a.ld_res, size)) || (a.res_out && !on16(a.res_out, a.ld_res_out, size))) return false;
    if ((a.dout && !on16(a.dout, a.ld_dout, size)) || (a.dres && !on16(a.dres, a.ld_dres, size)) || (a.dx && !on16(a.dx, a.ld_dx, size))) return false;
    if (!a.out) return true;
    const int out_size = a.out_dtype == GEAR_E4M3 ? 1 : a.out_dtype == GEAR_BF16 ? 2 : 4;
    return on16(a.out, a.ld_out, out_size);
}

template <typename T, bool VEC, int W, int C> static cudaError_t norm_go(const NormArgs& a, cudaStream_t st) {
    constexpr int ROWS = W == 1 ? NORM_WARPS : 1;
    return launch_dependent(rms_norm_kernel<T, VEC, W, C>, dim3((unsigned)ceil_div(a.n, ROWS)), dim3(32 * (W == 1 ? NORM_WARPS : W)), 0, st, a);
}
// rows up to this many columns stay in a warp's registers; up to eight times that, in a block's
constexpr int WARP_COLS = 2048;

template <typename T, bool VEC> static cudaError_t norm_by_width(const NormArgs& a, cudaStream_t st) {
    constexpr int COLS = Chunk<T, VEC>::COLS, C = WARP_COLS / COLS;
    // few rows: all eight warps of a block on a row, which then waits for a fraction of the loads
    const bool few = a.n < (int64_t)sm_count() * 8 && a.cols > COLS;
    if (few && a.cols <= WARP_COLS) return norm_go<T, VEC, 8, (C + 7) / 8>(a, st);
    if (a.cols <= WARP_COLS / 4) return norm_go<T, VEC, 1, C / 4>(a, st);
    if (a.cols <= WARP_COLS) return norm_go<T, VEC, 1, C>(a, st);
    if (a.cols <= 8 * WARP_COLS / 2) return norm_go<T, VEC, 8, C / 2>(a, st);
    const int64_t blocks = a.n < (int64_t)sm_count() * 8 ? a.n : (int64_t)sm_count() * 8;
    return launch_dependent(rms_norm_wide_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, a);
}

template <typename T, bool VEC, int W, int C> static cudaError_t back_go(const NormArgs& a, int* blocks, cudaStream_t st) {
    constexpr int ROWS = W == 1 ? NORM_WARPS : 1;
    const int64_t want = ceil_div(a.n, ROWS);
    *blocks = (int)(want < GEAR_NORM_WORKSPACE_ROWS ? want : GEAR_NORM_WORKSPACE_ROWS);
    return launch_dependent(rms_norm_back_kernel<T, VEC, W, C>, dim3((unsigned)*blocks), dim3(32 * (W == 1 ? NORM_WARPS : W)),
                            W == 1 ? (size_t)a.cols * 4 : 0, st, a);
}
template <typename T, bool VEC> static cudaError_t back_by_width(const NormArgs& a, int* blocks, cudaStream_t st) {
    constexpr int COLS = Chunk<T, VEC>::COLS, C = WARP_COLS / COLS;
    const bool few = a.n < (int64_t)sm_count() * 8 && a.cols > COLS;
    if (few && a.cols <= WARP_COLS) return back_go<T, VEC, 8, (C + 7) / 8>(a, blocks, st);
    if (a.cols <= WARP_COLS / 4) return back_go<T, VEC, 1, C / 4>(a, blocks, st);
    if (a.cols <= WARP_COLS) return back_go<T, VEC, 8, (C + 7) / 8>(a, blocks, st);
    if (a.cols <= 8 * WARP_COLS / 2) return back_go<T, VEC, 8, C / 2>(a, blocks, st);
    *blocks = (int)(a.n < GEAR_NORM_WORKSPACE_ROWS ? a.n : GEAR_NORM_WORKSPACE_ROWS);
    return launch_dependent(rms_norm_back_wide_kernel<T>, dim3((unsigned)*blocks), dim3(256), 0, st, a);
}

cudaError_t launch_rms_norm(const NormArgs& a, int dtype, cudaStream_t st) {
    if (a.n <= 0) return cudaSuccess;
    if (dtype == GEAR_BF16) return vectors(a, 2) ? norm_by_width<__nv_bfloat16, true>(a, st) : norm_by_width<__nv_bfloat16, false>(a, st);
    return vectors(a, 4) ? norm_by_width<float, true>(a, st) : norm_by_width<float, false>(a, st);
}

cudaError_t launch_rms_norm_backward(const NormArgs& a, int dtype, cudaStream_t st) {
    if (a.n <= 0) return a.dweight ? enqueue_memset(a.dweight, (size_t)a.cols * 4, st) : cudaSuccess;
    int blocks = 0;
    cudaError_t e;
    if (dtype == GEAR_BF16) e = vectors(a, 2) ? back_by_width<__nv_bfloat16, true>(a, &blocks, st) : back_by_width<__nv_bfloat16, false>(a, &blocks, st);
    else e = vectors(a, 4) ? back_by_width<float, true>(a, &blocks, st) : back_by_width<float, false>(a, &blocks, st);
    if (e != cudaSuccess || !a.dweight) return e;
    return launch_dependent(norm_dweight_kernel, dim3((unsigned)ceil_div(a.cols, 32)), dim3(256), 0, st, static_cast<const float*>(a.parts), blocks,
                            a.cols, a.dweight);
}

cudaError_t launch_q8_weights(const float* W, int64_t ldw, int K, int N, uint8_t* q, int64_t ldq, float* scale, uint8_t* qt, int64_t ldqt,
                              float* scale_t, cudaStream_t st) {
    constexpr int SMEM = Q8_BLOCK * (Q8_BLOCK + 1) * 4;
    if (const cudaError_t e = allow_smem<q8_weights_kernel>(SMEM)) return e;
    return launch_dependent(q8_weights_kernel, dim3((unsigned)ceil_div(K, Q8_BLOCK), (unsigned)ceil_div(N, Q8_BLOCK)), dim3(256), (size_t)SMEM, st,
                            W, ldw, K, N, q, ldq, scale, qt, ldqt, scale_t);
}

}  // namespace gear
