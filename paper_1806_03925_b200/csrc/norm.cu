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
#include <string.h>

#include <type_traits>

#include "internal.h"
#include "q8.cuh"

namespace gear {

// One lane's part of a chunk of columns that a warp holds.  VEC: E consecutive values in one load; else the lane has every 32nd value
// (any alignment, any width; a warp's loads are still whole lines).
template <typename T, bool VEC> struct Chunk;
template <> struct Chunk<float, true> {
    static constexpr int E = 4, COLS = 128;          // values, columns of the chunk
    float4 v;
    static __device__ __forceinline__ int col(int lane, int e) { return lane * 4 + e; }
    static __device__ __forceinline__ bool in(int lane, int, int left) { return lane * 4 < left; }      // (widths are multiples of E)
    __device__ __forceinline__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p, int lane, int left) { if (lane * 4 < left) v = *reinterpret_cast<const float4*>(p + lane * 4); else zero(); }
    __device__ __forceinline__ void store(float* p, int lane, int left) const { if (lane * 4 < left) *reinterpret_cast<float4*>(p + lane * 4) = v; }
    __device__ __forceinline__ void add(const Chunk& r) { v.x += r.v.x; v.y += r.v.y; v.z += r.v.z; v.w += r.v.w; }
    __device__ __forceinline__ void get(f32x2 (&f)[2]) const { f[0] = pack2(v.x, v.y); f[1] = pack2(v.z, v.w); }
    __device__ __forceinline__ void set(const f32x2 (&f)[2]) { v = make_float4(low(f[0]), high(f[0]), low(f[1]), high(f[1])); }
};
template <> struct Chunk<__nv_bfloat16, true> {
    static constexpr int E = 8, COLS = 256;
    uint4 v;
    static __device__ __forceinline__ int col(int lane, int e) { return lane * 8 + e; }
    static __device__ __forceinline__ bool in(int lane, int, int left) { return lane * 8 < left; }
    __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int lane, int left) { if (lane * 8 < left) v = *reinterpret_cast<const uint4*>(p + lane * 8); else zero(); }
    __device__ __forceinline__ void store(__nv_bfloat16* p, int lane, int left) const { if (lane * 8 < left) *reinterpret_cast<uint4*>(p + lane * 8) = v; }
    __device__ __forceinline__ void add(const Chunk& r) {      // (each sum rounded once)
        asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(r.v.x)); asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(r.v.y));
        asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v.z) : "r"(r.v.z)); asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(v.w) : "r"(r.v.w));
    }
    __device__ __forceinline__ void get(f32x2 (&f)[4]) const { f[0] = from_bf16x2(v.x); f[1] = from_bf16x2(v.y); f[2] = from_bf16x2(v.z); f[3] = from_bf16x2(v.w); }
    __device__ __forceinline__ void set(const f32x2 (&f)[4]) { v = make_uint4(to_bf16x2(f[0]), to_bf16x2(f[1]), to_bf16x2(f[2]), to_bf16x2(f[3])); }
};
template <typename T> struct Chunk<T, false> {
    static constexpr int E = 4, COLS = 128;
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
    __device__ __forceinline__ void add(const Chunk& r) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = v[e] + r.v[e];
    }
    __device__ __forceinline__ void get(f32x2 (&f)[2]) const { f[0] = pack2((float)v[0], (float)v[1]); f[1] = pack2((float)v[2], (float)v[3]); }
    __device__ __forceinline__ void set(const f32x2 (&f)[2]) { v[0] = (T)low(f[0]); v[1] = (T)high(f[0]); v[2] = (T)low(f[1]); v[3] = (T)high(f[1]); }
};

__device__ __forceinline__ float half_of(f32x2 v, int e) { return e & 1 ? high(v) : low(v); }

// A lane's values of a vector of weights (null: ones)
template <bool VEC, int H> __device__ __forceinline__ void load_weight(const float* w, int lane, int left, f32x2 (&f)[H]) {
    if (w == nullptr) {
#pragma unroll
        for (int e = 0; e < H; ++e) f[e] = both(1.f);
    } else if (VEC) {
#pragma unroll
        for (int e = 0; e < H; e += 2) {
            const float4 v = lane * 2 * H + 2 * e < left ? __ldg(reinterpret_cast<const float4*>(w + lane * 2 * H + 2 * e)) : make_float4(0.f, 0.f, 0.f, 0.f);
            f[e] = pack2(v.x, v.y); f[e + 1] = pack2(v.z, v.w);
        }
    } else {
#pragma unroll
        for (int e = 0; e < H; ++e)
            f[e] = pack2(lane + 64 * e < left ? __ldg(w + lane + 64 * e) : 0.f, lane + 64 * e + 32 < left ? __ldg(w + lane + 64 * e + 32) : 0.f);
    }
}

// The largest magnitude of the block that a lane's values belong to.  The whole warp calls.
template <bool VEC, int H> __device__ __forceinline__ float block_largest(const f32x2 (&v)[H], int lane) {
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < H; ++e) most = q8_larger(most, low(v[e]), high(v[e]));
    if (VEC && H == 4) {                         // half a warp a block
        const uint32_t m = __float_as_uint(most);
        const uint32_t a = __reduce_max_sync(0xffffffffu, lane < 16 ? m : 0u), b = __reduce_max_sync(0xffffffffu, lane < 16 ? 0u : m);
        return __uint_as_float(lane < 16 ? a : b);
    }
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
}
// A lane's values in e4m3 to a row; quotient: what becomes of a pair
template <bool VEC, int H, typename Fn> __device__ __forceinline__ void put_q8(uint8_t* q, int lane, int left, const f32x2 (&v)[H], const Fn& quotient) {
    uint32_t w[H / 2];
#pragma unroll
    for (int e = 0; e < H; e += 2) w[e / 2] = (uint32_t)q8_pair(quotient(v[e])) | (uint32_t)q8_pair(quotient(v[e + 1])) << 16;
    if (VEC) {
        if (lane * 2 * H < left) {
            if (H == 2) *reinterpret_cast<uint32_t*>(q + lane * 4) = w[0];
            else *reinterpret_cast<uint2*>(q + lane * 8) = make_uint2(w[0], w[H / 2 - 1]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) if (lane + 32 * e < left) q[lane + 32 * e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
    }
}
// The piece's values before r is known, if its block is a usual one; returns the block's largest.
template <bool VEC, int H> __device__ __forceinline__ float put_q8_early(void* row, int col0, int lane, int left, const f32x2 (&v)[H]) {
    const float largest = block_largest<VEC>(v, lane);
    if (q8_usual(largest)) put_q8<VEC>(static_cast<uint8_t*>(row) + col0, lane, left, v, Q8Quotient(largest));
    return largest;
}
// A lane's values, times r, to a row of fp32 or bf16.
template <bool VEC, int H> __device__ __forceinline__ void put_row(void* row, int col0, int lane, int left, int dtype, float r, f32x2 (&h)[H]) {
    const bool in = lane * 2 * H < left;                              // (VEC: all of the lane's values or none)
#pragma unroll
    for (int e = 0; e < H; ++e) h[e] = mul2(h[e], both(r));
    if (dtype == GEAR_BF16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(row) + col0;
        uint32_t w[H];
#pragma unroll
        for (int e = 0; e < H; ++e) w[e] = to_bf16x2(h[e]);
        if (VEC) {
            if (in) {
                if (H == 2) *reinterpret_cast<uint2*>(o + lane * 4) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint4*>(o + lane * 8) = make_uint4(w[0], w[1], w[H - 2], w[H - 1]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 2 * H; ++e) if (lane + 32 * e < left) o[lane + 32 * e] = __ushort_as_bfloat16((unsigned short)(w[e / 2] >> (16 * (e % 2))));
        }
    } else {
        float* o = static_cast<float*>(row) + col0;
        if (VEC) {
            if (in)
#pragma unroll
                for (int e = 0; e < H; e += 2) *reinterpret_cast<float4*>(o + lane * 2 * H + 2 * e) = make_float4(low(h[e]), high(h[e]), low(h[e + 1]), high(h[e + 1]));
        } else {
#pragma unroll
            for (int e = 0; e < H; ++e) {
                if (lane + 64 * e < left) o[lane + 64 * e] = low(h[e]);
                if (lane + 64 * e + 32 < left) o[lane + 64 * e + 32] = high(h[e]);
            }
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

// A piece of row k written by the definition, where its block is not a usual one: y is read again, from res_out if it has been kept there,
// else made again.  (Out of line: divisions for every value in every piece of a row would be most of the kernel's instructions.)
template <typename T, bool VEC>
__device__ __noinline__ void q8_by_definition(const NormArgs& a, int64_t k, int col0, int lane, float largest, float r) {
    typedef Chunk<T, VEC> Ch;
    constexpr int H = Ch::E / 2;
    const int left = a.cols - col0;
    Ch y;
    if (a.res_out) y.load(static_cast<const T*>(a.res_out) + k * a.ld_res_out + col0, lane, left);
    else {
        const T* x = row_of_x<T>(a, k, false);
        if (x) y.load(x + col0, lane, left); else y.zero();
        if (a.res) {
            Ch s;
            s.load(static_cast<const T*>(a.res) + k * a.ld_res + col0, lane, left);
            y.add(s);
        }
    }
    f32x2 v[H];
    y.get(v);
    if (a.weight) {
        f32x2 w[H];
        load_weight<VEC, H>(a.weight + col0, lane, left, w);
#pragma unroll
        for (int e = 0; e < H; ++e) v[e] = mul2(v[e], w[e]);
    }
    put_q8<VEC>(static_cast<uint8_t*>(row_of_out<T>(a, k)) + col0, lane, left, v, Q8Plain(largest, r));
}
// The scales of a piece's blocks, once r is known.
template <typename T, bool VEC> __device__ __forceinline__ void put_q8_late(const NormArgs& a, int64_t k, float* scales, int col0, int lane, float largest, float r) {
    constexpr int LANES = VEC && Chunk<T, VEC>::E == 8 ? 16 : 32;     // lanes that share a block
    float s = q8_usual_scale(largest, r);
    if (!q8_usual(largest, r)) {
        q8_by_definition<T, VEC>(a, k, col0, lane, largest, r);
        s = Q8Plain(largest, r).scale;
    }
    if (lane % LANES == 0 && col0 + (lane / LANES) * Q8_BLOCK < a.cols) scales[col0 / Q8_BLOCK + lane / LANES] = s;
}

// v summed over the warps that share a row; scratch: a word for each.  (All warps of the block call.)
__device__ __forceinline__ float sum_over_row(float v, float* scratch, int part, int warps) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) scratch[part] = v;
    __syncthreads();
    float t = 0.f;
    for (int w = 0; w < warps; ++w) t += scratch[w];
    return t;
}

constexpr int NORM_ROWS = 4;                     // rows per block where a warp has a row of its own

// A row to a warp (ONE) or to all warps of a block; C pieces of columns a warp: piece c * warps + part.
template <typename T, bool VEC, bool ONE, int C>
__global__ void __launch_bounds__(ONE ? 32 * NORM_ROWS : 256)
rms_norm_kernel(const __grid_constant__ NormArgs a) {
    typedef Chunk<T, VEC> Ch;
    constexpr int H = Ch::E / 2;
    __shared__ float scratch[8];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = ONE ? 0 : warp, warps = ONE ? 1 : blockDim.x >> 5;
    const int64_t k = ONE ? (int64_t)blockIdx.x * NORM_ROWS + warp : (int64_t)blockIdx.x;
    if (k >= live_rows(a)) return;               // (uniform over the warps of a row)
    const T* x = row_of_x<T>(a, k, lane == 0 && part == 0);
    auto first = [&](int c) { return (c * warps + part) * Ch::COLS; };
    Ch y[C];
#pragma unroll
    for (int c = 0; c < C; ++c) { if (x) y[c].load(x + first(c), lane, a.cols - first(c)); else y[c].zero(); }
    if (a.res) {
        const T* res = static_cast<const T*>(a.res) + k * a.ld_res;
        Ch r[C];
#pragma unroll
        for (int c = 0; c < C; ++c) r[c].load(res + first(c), lane, a.cols - first(c));
#pragma unroll
        for (int c = 0; c < C; ++c) y[c].add(r[c]);      // the residual stream is kept in its own type; the norm is the kept sum's
    }
    if (a.res_out) {
        T* o = static_cast<T*>(a.res_out) + k * a.ld_res_out;
#pragma unroll
        for (int c = 0; c < C; ++c) y[c].store(o + first(c), lane, a.cols - first(c));
    }
    void* out = row_of_out<T>(a, k);
    const bool q8 = a.out_dtype == GEAR_E4M3;
    auto value = [&](int c, f32x2 (&v)[H]) {     // y times the weights
        y[c].get(v);
        if (a.weight) {
            f32x2 w[H];
            load_weight<VEC, H>(a.weight + first(c), lane, a.cols - first(c), w);
#pragma unroll
            for (int e = 0; e < H; ++e) v[e] = mul2(v[e], w[e]);
        }
    };
    float largest[C];
    f32x2 sum2 = 0ull;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (first(c) >= a.cols) continue;
        f32x2 v[H];
        if (a.normed) {
            y[c].get(v);
#pragma unroll
            for (int e = 0; e < H; ++e) sum2 = fma2(v[e], v[e], sum2);
        }
        if (q8) { value(c, v); largest[c] = put_q8_early<VEC, H>(out, first(c), lane, a.cols - first(c), v); }
    }
    float r = 1.f;
    if (a.normed) {
        float sum = low(sum2) + high(sum2);
        sum = ONE ? warp_sum(sum) : sum_over_row(sum, scratch, part, warps);
        r = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col0 = first(c);
        if (col0 >= a.cols) continue;
        if (q8) put_q8_late<T, VEC>(a, k, a.scale + k * a.blocks, col0, lane, largest[c], r);
        else {
            f32x2 v[H];
            value(c, v);
            put_row<VEC, H>(out, col0, lane, a.cols - col0, a.out_dtype, r, v);
        }
    }
}

// Rows of any width: eight warps per row, three passes over it.
template <typename T>
__global__ void __launch_bounds__(256)
rms_norm_wide_kernel(const __grid_constant__ NormArgs a) {
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
        auto get = [&](int col0, bool from_kept, f32x2 (&f)[Ch::E / 2]) {
            Ch y;
            if (from_kept) { y.load(kept + col0, lane, a.cols - col0); y.get(f); return; }
            if (x) y.load(x + col0, lane, a.cols - col0); else y.zero();
            if (res) {
                Ch r;
                r.load(res + col0, lane, a.cols - col0);
                y.add(r);
            }
            y.get(f);
            if (kept) y.store(kept + col0, lane, a.cols - col0);
        };
        f32x2 sum2 = 0ull;
        if (a.normed || kept)
            for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
                f32x2 f[Ch::E / 2];
                get(col0, false, f);
#pragma unroll
                for (int e = 0; e < Ch::E / 2; ++e) sum2 = fma2(f[e], f[e], sum2);
            }
        const float sum = sum_over_row(low(sum2) + high(sum2), scratch, part, 8);
        const float r = a.normed ? 1.0f / sqrtf(sum / (float)a.cols + a.eps) : 1.f;
        void* out = row_of_out<T>(a, k);
        for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
            constexpr int H = Ch::E / 2;
            auto value = [&](f32x2 (&v)[H]) {
                get(col0, kept != nullptr, v);
                if (a.weight) {
                    f32x2 w[H];
                    load_weight<false, H>(a.weight + col0, lane, a.cols - col0, w);
#pragma unroll
                    for (int e = 0; e < H; ++e) v[e] = mul2(v[e], w[e]);
                }
            };
            f32x2 v[H];
            value(v);
            if (a.out_dtype == GEAR_E4M3) {
                const float largest = put_q8_early<false, H>(out, col0, lane, a.cols - col0, v);
                put_q8_late<T, false>(a, k, a.scale + k * a.blocks, col0, lane, largest, r);
            } else put_row<false, H>(out, col0, lane, a.cols - col0, a.out_dtype, r, v);
        }
        __syncthreads();                         // scratch is free for the next row
    }
}

// ---------------------------------------------------------------- gradients
// A row to a block, a lane the same C pieces of columns of every row: it keeps its weights and its part of dw in registers for as long as
// it lives.  The next row is on its way while the warps meet over one row's sums.  At the end the block's part of dw goes to its row
// of `parts`.  Nothing is added up in an order that could change.
template <typename T, bool VEC, int C, int PER_SM>
__global__ void __launch_bounds__(256, PER_SM)
rms_norm_back_kernel(const NormArgs a) {
    typedef Chunk<T, VEC> Ch;
    constexpr int H = Ch::E / 2;
    __shared__ float2 scratch[2][8];             // two sets in turn: a row's sums are read by all before those of the row after the next are written
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t live = live_rows(a);
    const float inv_cols = 1.0f / (float)a.cols;
    f32x2 w[C][H], dw[C][H];
    auto first = [&](int c) { return (c * warps + warp) * Ch::COLS; };
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_weight<VEC, H>(a.weight && first(c) < a.cols ? a.weight + first(c) : nullptr, lane, a.cols - first(c), w[c]);
#pragma unroll
        for (int e = 0; e < H; ++e) dw[c][e] = 0ull;
    }
    Ch y[C], g[C], s[C];
    auto fetch = [&](int64_t k) {
        const T* x = row_of_x<T>(a, k, threadIdx.x == 0);
        const T* dout = static_cast<const T*>(a.dout) + k * a.ld_dout;
        const T* dres = a.dres ? static_cast<const T*>(a.dres) + k * a.ld_dres : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (x) y[c].load(x + first(c), lane, a.cols - first(c)); else y[c].zero();
            g[c].load(dout + first(c), lane, a.cols - first(c));
            if (dres) s[c].load(dres + first(c), lane, a.cols - first(c)); else s[c].zero();
        }
    };
    int odd = 0;
    int64_t k = blockIdx.x;
    if (k < live) fetch(k);
    for (; k < live; k += gridDim.x, odd ^= 1) {
        Ch y0[C], g0[C], s0[C];
        f32x2 sq = 0ull, dot = 0ull;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            y0[c] = y[c]; g0[c] = g[c]; s0[c] = s[c];
            f32x2 f[H], d[H];
            y0[c].get(f); g0[c].get(d);
#pragma unroll
            for (int e = 0; e < H; ++e) { sq = fma2(f[e], f[e], sq); dot = fma2(mul2(d[e], w[c][e]), f[e], dot); }
        }
        if (k + gridDim.x < live) fetch(k + gridDim.x);
        float2 sum = make_float2(warp_sum(low(sq) + high(sq)), warp_sum(low(dot) + high(dot)));
        if (warps > 1) {
            if (lane == 0) scratch[odd][warp] = sum;
            __syncthreads();
            sum = make_float2(0.f, 0.f);
            for (int v = 0; v < warps; ++v) { sum.x += scratch[odd][v].x; sum.y += scratch[odd][v].y; }
        }
        const float r = 1.0f / sqrtf(sum.x * inv_cols + a.eps);
        const float q = r * (r * (sum.y * inv_cols));          // dx = r (g - y q): r alone may be large where y is small, and r r not a number
#pragma unroll
        for (int c = 0; c < C; ++c) {
            f32x2 f[H], d[H], o[H];
            y0[c].get(f); g0[c].get(d); s0[c].get(o);
#pragma unroll
            for (int e = 0; e < H; ++e) {
                o[e] = fma2(both(r), fma2(f[e], both(-q), mul2(d[e], w[c][e])), o[e]);
                dw[c][e] = fma2(mul2(d[e], both(r)), f[e], dw[c][e]);
            }
            if (a.dx) {
                s0[c].set(o);
                s0[c].store(static_cast<T*>(a.dx) + k * a.ld_dx + first(c), lane, a.cols - first(c));
            }
        }
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < Ch::E; ++e) if (Ch::in(lane, e, a.cols - first(c))) to[first(c) + Ch::col(lane, e)] = half_of(dw[c][e / 2], e);
}

// Narrow rows: a warp has rows of its own, one grid's warps apart, and the next one on its way into shared memory while it works on
// one: a lane copies (16 bytes at a time) the very pieces it will read, so that nobody waits for anybody.
constexpr int STREAM = 2, STREAM_WARPS = 4;
constexpr int stream_smem(int arrays, int C) { return STREAM_WARPS * STREAM * arrays * C * 512; }

// The pieces of row `row` (null: zeros) to the lane's places at `smem`.
template <typename T, int C> __device__ __forceinline__ void stream_row(uint32_t smem, const T* row, const T* any, int lane, int cols) {
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = c * 32 * E + lane * E;
        const bool there = row != nullptr && col < cols;
        cp_async_16(smem + (uint32_t)(c * 512 + lane * 16), there ? row + col : any, there ? 16 : 0);
    }
}
template <typename T, typename Ch> __device__ __forceinline__ void take_piece(Ch& ch, uint32_t smem, int c, int lane) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem + (uint32_t)(c * 512 + lane * 16)) : "memory");
    memcpy(&ch.v, &v, 16);
}

// A row is read from shared memory twice (sums, results), so
// that registers hold little but the warp's part of dw; at the end the warps of a block add theirs up one after the other.
template <typename T, int C, bool RES>
__global__ void __launch_bounds__(32 * STREAM_WARPS)
rms_norm_back_stream_kernel(const NormArgs a) {
    typedef Chunk<T, true> Ch;
    constexpr int ARRAYS = RES ? 3 : 2;
    extern __shared__ __align__(16) uint8_t stream_mem[];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(stream_mem) + (uint32_t)(warp * STREAM * ARRAYS * C * 512);
    const int64_t live = live_rows(a), step = (int64_t)gridDim.x * STREAM_WARPS;
    const T *any = static_cast<const T*>(a.x), *dout = static_cast<const T*>(a.dout), *dres = static_cast<const T*>(a.dres);
    const float inv_cols = 1.0f / (float)a.cols;
    int64_t next = (int64_t)blockIdx.x * STREAM_WARPS + warp;
    int next_slot = 0;
    auto send = [&] {
        if (next < live) {
            const uint32_t at = mine + (uint32_t)(next_slot * ARRAYS * C * 512);
            stream_row<T, C>(at, row_of_x<T>(a, next, lane == 0), any, lane, a.cols);
            stream_row<T, C>(at + C * 512, dout + next * a.ld_dout, dout, lane, a.cols);
            if (RES) stream_row<T, C>(at + 2 * C * 512, dres + next * a.ld_dres, dres, lane, a.cols);
        }
        cp_async_commit();
        next += step;
        next_slot = next_slot == STREAM - 1 ? 0 : next_slot + 1;
    };
    f32x2 dw[C][Ch::E / 2];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < Ch::E / 2; ++e) dw[c][e] = 0ull;
    for (int d = 0; d < STREAM - 1; ++d) send();
    int slot = 0;
    for (int64_t k = (int64_t)blockIdx.x * STREAM_WARPS + warp; k < live; k += step) {
        send();
        cp_async_wait<STREAM - 1>();
        const uint32_t at = mine + (uint32_t)(slot * ARRAYS * C * 512);
        slot = slot == STREAM - 1 ? 0 : slot + 1;
        f32x2 sq2 = 0ull, dot2 = 0ull;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (c * Ch::COLS >= a.cols) continue;
            Ch y, g;
            f32x2 f[Ch::E / 2], d[Ch::E / 2], w[Ch::E / 2];
            take_piece<T>(y, at, c, lane); take_piece<T>(g, at + C * 512, c, lane);
            y.get(f); g.get(d);
            load_weight<true, Ch::E / 2>(a.weight ? a.weight + c * Ch::COLS : nullptr, lane, a.cols - c * Ch::COLS, w);
#pragma unroll
            for (int e = 0; e < Ch::E / 2; ++e) { sq2 = fma2(f[e], f[e], sq2); dot2 = fma2(mul2(d[e], w[e]), f[e], dot2); }
        }
        const float sq = warp_sum(low(sq2) + high(sq2)), dot = warp_sum(low(dot2) + high(dot2));
        const float r = 1.0f / sqrtf(sq * inv_cols + a.eps);
        const float q = r * (r * (dot * inv_cols));
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = a.cols - c * Ch::COLS;
            if (left <= 0) continue;
            Ch y, g, s;
            f32x2 f[Ch::E / 2], d[Ch::E / 2], w[Ch::E / 2], o[Ch::E / 2];
            take_piece<T>(y, at, c, lane); take_piece<T>(g, at + C * 512, c, lane);
            if (RES) take_piece<T>(s, at + 2 * C * 512, c, lane); else s.zero();
            y.get(f); g.get(d); s.get(o);
            load_weight<true, Ch::E / 2>(a.weight ? a.weight + c * Ch::COLS : nullptr, lane, left, w);
#pragma unroll
            for (int e = 0; e < Ch::E / 2; ++e) {
                o[e] = fma2(both(r), fma2(f[e], both(-q), mul2(d[e], w[e])), o[e]);
                dw[c][e] = fma2(mul2(d[e], both(r)), f[e], dw[c][e]);
            }
            if (a.dx) {
                s.set(o);
                s.store(static_cast<T*>(a.dx) + k * a.ld_dx + c * Ch::COLS, lane, left);
            }
        }
    }
    cp_async_wait<0>();
    if (!a.parts) return;
    float* sum = reinterpret_cast<float*>(stream_mem);
    for (int turn = 0; turn < STREAM_WARPS; ++turn) {
        __syncthreads();
        if (warp == turn)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < Ch::E; ++e) {
                    const int col = c * Ch::COLS + Ch::col(lane, e);
                    if (col < a.cols) sum[col] = turn == 0 ? half_of(dw[c][e / 2], e) : sum[col] + half_of(dw[c][e / 2], e);
                }
    }
    __syncthreads();
    for (int col = threadIdx.x; col < a.cols; col += 32 * STREAM_WARPS) a.parts[(int64_t)blockIdx.x * a.cols + col] = sum[col];
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
        f32x2 sq2 = 0ull, dot2 = 0ull;
        for (int pass = 0; pass < 2; ++pass) {
            const float inv_cols = 1.0f / (float)a.cols;
            const float r = 1.0f / sqrtf(sq * inv_cols + a.eps), q = r * (r * (dot * inv_cols));    // (second pass)
            for (int col0 = part * Ch::COLS; col0 < a.cols; col0 += 8 * Ch::COLS) {
                const int left = a.cols - col0;
                Ch y, g;
                f32x2 f[Ch::E / 2], d[Ch::E / 2], w[Ch::E / 2], o[Ch::E / 2];
                if (x) y.load(x + col0, lane, left); else y.zero();
                g.load(dout + col0, lane, left);
                y.get(f); g.get(d);
                load_weight<false, Ch::E / 2>(a.weight ? a.weight + col0 : nullptr, lane, left, w);
                if (pass == 0) {
#pragma unroll
                    for (int e = 0; e < Ch::E / 2; ++e) { sq2 = fma2(f[e], f[e], sq2); dot2 = fma2(mul2(d[e], w[e]), f[e], dot2); }
                    continue;
                }
                if (a.dx) {
#pragma unroll
                    for (int e = 0; e < Ch::E / 2; ++e) o[e] = mul2(both(r), fma2(f[e], both(-q), mul2(d[e], w[e])));
                    Ch s;
                    if (a.dres) {
                        f32x2 t[Ch::E / 2];
                        s.load(static_cast<const T*>(a.dres) + k * a.ld_dres + col0, lane, left);
                        s.get(t);
#pragma unroll
                        for (int e = 0; e < Ch::E / 2; ++e) o[e] = add2(o[e], t[e]);
                    }
                    s.set(o);
                    s.store(static_cast<T*>(a.dx) + k * a.ld_dx + col0, lane, left);
                }
                if (to)
#pragma unroll
                    for (int e = 0; e < Ch::E; ++e)
                        if (Ch::in(lane, e, left)) { float* p = to + col0 + Ch::col(lane, e); *p = fmaf(half_of(d[e / 2], e) * r, half_of(f[e / 2], e), *p); }
            }
            if (pass == 0) { sq = sum_over_row(low(sq2) + high(sq2), scratch[0], part, 8); dot = sum_over_row(low(dot2) + high(dot2), scratch[1], part, 8); }
        }
        __syncthreads();
    }
}

// dw[c] = the blocks' sums added up, always in the same order: 32 columns a block, 32 warps over the rows, eight rows on their way
// at a time (with eight warps and one row: as long as the rest of the call for 3001 rows of 1001)
__global__ void __launch_bounds__(1024)
norm_dweight_kernel(const float* __restrict__ parts, int rows, int cols, float* __restrict__ dweight) {
    __shared__ float s[32][33];
    wait_for_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float t = 0.f;
    if (col < cols)
        for (int r0 = warp; r0 < rows; r0 += 32 * 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r0 + 32 * i < rows ? __ldcg(parts + (int64_t)(r0 + 32 * i) * cols + col) : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) t += v[i];
        }
    s[warp][lane] = t;
    __syncthreads();
    t = warp_sum(s[lane][warp]);                 // warp w adds up column w
    if (lane == 0 && blockIdx.x * 32 + warp < cols) dweight[blockIdx.x * 32 + warp] = t;
}

// ---------------------------------------------------------------- weights
// One block per 128 x 128 weights.  A lane holds squares of 4 x 4 of them from their load on: its values of a row are four bytes of the
// transposed copy, and, turned round in registers, four bytes of a column go to shared memory, from where whole rows of the other copy
// leave.  (The weights as fp32 in shared memory, bytes stored one by one: 10.1 us for 2048 x 1024, this 4.1.)
constexpr int QW_THREADS = 512;
__device__ __forceinline__ void put_bytes(uint8_t* p, uint32_t w, int left, bool words) {
    if (words && left >= 4) *reinterpret_cast<uint32_t*>(p) = w;
    else
        for (int i = 0; i < 4 && i < left; ++i) p[i] = (uint8_t)(w >> (8 * i));
}
__global__ void __launch_bounds__(QW_THREADS)
q8_weights_kernel(const float* __restrict__ W, int64_t ldw, int vec, int K, int N, uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale,
                  uint8_t* __restrict__ qt, int64_t ldqt, float* __restrict__ scale_t) {
    __shared__ uint32_t turned[Q8_BLOCK][33];    // [column][four rows]
    __shared__ uint32_t most[QW_THREADS / 32];
    wait_for_predecessor();
    constexpr int SQUARES = Q8_BLOCK / 4 / (QW_THREADS / 32);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // (one number for both: a grid's second dimension ends at 65535)
    const unsigned k_blocks = (unsigned)(K + Q8_BLOCK - 1) / Q8_BLOCK, n_blocks = (unsigned)(N + Q8_BLOCK - 1) / Q8_BLOCK;
    const unsigned nb = blockIdx.x / k_blocks, kb = blockIdx.x - nb * k_blocks;
    const int k0 = (int)kb * Q8_BLOCK, n0 = (int)nb * Q8_BLOCK, kn = min(Q8_BLOCK, K - k0), nn = min(Q8_BLOCK, N - n0);
    float4 v[SQUARES][4];
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < SQUARES; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int k = 4 * (warp + i * (QW_THREADS / 32)) + r, n = 4 * lane;
            const float* p = W + (int64_t)(k0 + k) * ldw + n0 + n;
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k < kn) {
                if (vec && n + 4 <= nn) f = __ldg(reinterpret_cast<const float4*>(p));
                else {
                    if (n < nn) f.x = __ldg(p);
                    if (n + 1 < nn) f.y = __ldg(p + 1);
                    if (n + 2 < nn) f.z = __ldg(p + 2);
                    if (n + 3 < nn) f.w = __ldg(p + 3);
                }
            }
            v[i][r] = f;
        }
#pragma unroll
    for (int i = 0; i < SQUARES; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mine = q8_larger(q8_larger(mine, v[i][r].x, v[i][r].y), v[i][r].z, v[i][r].w);
    uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(mine));
    if (lane == 0) most[warp] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, most[lane & (QW_THREADS / 32 - 1)]);
    const float largest = __uint_as_float(m);
    const bool usual = q8_usual(largest, 1.f);
    const Q8Quotient fast(largest);
    const Q8Plain plain(largest, 1.f);
    if (threadIdx.x == 0) {
        const float s = usual ? q8_usual_scale(largest, 1.f) : plain.scale;
        if (q) scale[(int64_t)nb * k_blocks + kb] = s;
        if (qt) scale_t[(int64_t)kb * n_blocks + nb] = s;
    }
    const bool words_t = (reinterpret_cast<uintptr_t>(qt) & 3u) == 0 && (ldqt & 3) == 0, words = (reinterpret_cast<uintptr_t>(q) & 3u) == 0 && (ldq & 3) == 0;
#pragma unroll
    for (int i = 0; i < SQUARES; ++i) {
        const int k4 = warp + i * (QW_THREADS / 32);
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const f32x2 a = pack2(v[i][r].x, v[i][r].y), b = pack2(v[i][r].z, v[i][r].w);
            w[r] = usual ? (uint32_t)q8_pair(fast(a)) | (uint32_t)q8_pair(fast(b)) << 16 : (uint32_t)q8_pair(plain(a)) | (uint32_t)q8_pair(plain(b)) << 16;
            if (qt && 4 * k4 + r < kn && 4 * lane < nn) put_bytes(qt + (int64_t)(k0 + 4 * k4 + r) * ldqt + n0 + 4 * lane, w[r], nn - 4 * lane, words_t);
        }
        const uint32_t a01 = __byte_perm(w[0], w[1], 0x5140), a23 = __byte_perm(w[2], w[3], 0x5140), b01 = __byte_perm(w[0], w[1], 0x7362), b23 = __byte_perm(w[2], w[3], 0x7362);
        turned[4 * lane][k4] = __byte_perm(a01, a23, 0x5410);
        turned[4 * lane + 1][k4] = __byte_perm(a01, a23, 0x7632);
        turned[4 * lane + 2][k4] = __byte_perm(b01, b23, 0x5410);
        turned[4 * lane + 3][k4] = __byte_perm(b01, b23, 0x7632);
    }
    if (!q) return;
    __syncthreads();
    for (int n = warp; n < nn; n += QW_THREADS / 32)
        if (4 * lane < kn) put_bytes(q + (int64_t)(n0 + n) * ldq + k0 + 4 * lane, turned[n][lane], kn - 4 * lane, words);
}

// ---------------------------------------------------------------- host side
static bool on16(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0; }

// whether all rows, 8-bit ones too, start on 16-byte boundaries and hold whole vectors of the input's type
static bool vectors(const NormArgs& a, int size) {
    const int64_t vec = 16 / size;
    if (a.cols % vec || !on16(a.x, a.ldx, size) || (a.weight && !on16(a.weight, 0, 4))) return false;
    if ((a.res && !on16(a.res, a.ld_res, size)) || (a.res_out && !on16(a.res_out, a.ld_res_out, size))) return false;
    if ((a.dout && !on16(a.dout, a.ld_dout, size)) || (a.dres && !on16(a.dres, a.ld_dres, size)) || (a.dx && !on16(a.dx, a.ld_dx, size))) return false;
    if (!a.out) return true;
    const int out_size = a.out_dtype == GEAR_E4M3 ? 1 : a.out_dtype == GEAR_BF16 ? 2 : 4;
    return on16(a.out, a.ld_out, out_size);
}

// A stream of rows to every warp: blocks of STREAM_WARPS warps, as many as an SM's shared memory takes (at most eight).  The rows
// have to be enough to fill the streams.
constexpr int64_t SMEM_PER_SM = 227 * 1024;
static int stream_blocks(int smem) { const int64_t n = SMEM_PER_SM / (smem + 1024); return (int)(n < 8 ? n : 8); }
static bool stream_fits(int64_t n, int blocks) { return n >= (int64_t)sm_count() * blocks * STREAM_WARPS * 2; }

// f(C) with the smallest C that holds the row; false: none does, or the row is better off with a block (below)
template <typename T, typename Fn> static bool stream_width(int cols, bool res, Fn&& fn) {
    const int pieces = (int)ceil_div((int64_t)cols * (int)sizeof(T), 512);
    if (pieces > (res ? 4 : 6)) return false;
    if (pieces <= 1) fn(std::integral_constant<int, 1>{});
    else if (pieces <= 2) fn(std::integral_constant<int, 2>{});
    else if (pieces <= 4) fn(std::integral_constant<int, 4>{});
    else fn(std::integral_constant<int, 6>{});
    return true;
}
// true: the rows go by streams, *e is the launch's result
template <typename T, int C, bool RES> static bool back_stream_go(const NormArgs& a, int* grid, cudaError_t* e, cudaStream_t st) {
    constexpr int SMEM = stream_smem(RES ? 3 : 2, C);
    int blocks = stream_blocks(SMEM);
    if (blocks > GEAR_NORM_WORKSPACE_ROWS / sm_count()) blocks = GEAR_NORM_WORKSPACE_ROWS / sm_count();
    if (blocks < 1 || !stream_fits(a.n, blocks)) return false;
    *grid = sm_count() * blocks;
    *e = allow_smem<rms_norm_back_stream_kernel<T, C, RES>>(SMEM);
    if (*e == cudaSuccess) *e = launch_now(rms_norm_back_stream_kernel<T, C, RES>, dim3((unsigned)*grid), dim3(32 * STREAM_WARPS), (size_t)SMEM, st, a);
    return true;
}
template <typename T> static bool back_stream(const NormArgs& a, int* grid, cudaError_t* e, cudaStream_t st) {
    bool went = false;
    stream_width<T>(a.cols, a.dres != nullptr, [&](auto c) { went = a.dres ? back_stream_go<T, decltype(c)::value, true>(a, grid, e, st) : back_stream_go<T, decltype(c)::value, false>(a, grid, e, st); });
    return went;
}

template <typename T, bool VEC, bool ONE, int C> static cudaError_t norm_go(const NormArgs& a, cudaStream_t st) {
    const int warps = ONE ? NORM_ROWS : (int)ceil_div(ceil_div(a.cols, Chunk<T, VEC>::COLS), C);
    return launch_now(rms_norm_kernel<T, VEC, ONE, C>, dim3((unsigned)(ONE ? ceil_div(a.n, NORM_ROWS) : a.n)), dim3(32 * warps), 0, st, a);
}
template <typename T, bool VEC> static cudaError_t norm_by_width(const NormArgs& a, cudaStream_t st) {
    constexpr int COLS = Chunk<T, VEC>::COLS;
    const int64_t pieces = ceil_div(a.cols, COLS);
    // Few rows: as many warps to a row as there are pieces, each of which then waits for its own loads alone.  Many: a row to a warp, and
    // what a warp does once is done once a row.  Wide rows in between: two pieces a warp.  e4m3 outputs, us, one piece / two pieces a warp / a
    // row to a warp.  bf16, 1536 columns, residual: 600 rows 3.2 / 3.5 / 5.8; 2500: 7.1 / 6.6 / 7.0; 12000: 30.0 / 25.4 / 30.8; 40000: 90.9 / 72.3 /
    // 74.9; 262144: 576 / 445 / 417.  fp32, 1536 columns by ID: 12000: - / 33.6 / 35.9; 40000: - / 102.9 / 94.6.  bf16, 500 columns: 600: 2.4 / 3.1 /
    // 3.9; 2500: 4.8 / 4.3 / 4.4; 12000: 16.2 / 13.3 / 11.7; 40000: 51.4 / 40.9 / 35.1.
    if (pieces == 1) return norm_go<T, VEC, true, 1>(a, st);
    if (pieces > 4 && pieces <= 16 && a.n >= 1024 && a.n < 24576) return norm_go<T, VEC, false, 2>(a, st);
    if (a.n >= 1024) {
        if (pieces <= 2) return norm_go<T, VEC, true, 2>(a, st);
        if (pieces <= 4) return norm_go<T, VEC, true, 4>(a, st);
        if (pieces <= 6) return norm_go<T, VEC, true, 6>(a, st);
        if (pieces <= 8) return norm_go<T, VEC, true, 8>(a, st);
        if constexpr (COLS == 128) {
            if (pieces <= 12) return norm_go<T, VEC, true, 12>(a, st);
            if (pieces <= 16) return norm_go<T, VEC, true, 16>(a, st);
        }
    }
    if (pieces <= 8) return norm_go<T, VEC, false, 1>(a, st);
    if (pieces <= 16) return norm_go<T, VEC, false, 2>(a, st);
    if (pieces <= 32) return norm_go<T, VEC, false, 4>(a, st);
    if constexpr (COLS == 128) { if (pieces <= 64) return norm_go<T, VEC, false, 8>(a, st); }
    const int64_t blocks = a.n < (int64_t)sm_count() * 8 ? a.n : (int64_t)sm_count() * 8;
    return launch_now(rms_norm_wide_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, a);
}

// PER_SM: blocks of 256 threads that an SM takes (in registers); the grid is no larger than what runs at once.
template <typename T, bool VEC, int C, int PER_SM> static cudaError_t back_go(const NormArgs& a, int* blocks, cudaStream_t st) {
    const int64_t most = (int64_t)sm_count() * PER_SM;
    *blocks = (int)(a.n < most ? a.n : most);
    if (*blocks > GEAR_NORM_WORKSPACE_ROWS) *blocks = GEAR_NORM_WORKSPACE_ROWS;
    const int warps = (int)ceil_div(ceil_div(a.cols, Chunk<T, VEC>::COLS), C);
    return launch_now(rms_norm_back_kernel<T, VEC, C, PER_SM>, dim3((unsigned)*blocks), dim3(32 * warps), 0, st, a);
}
template <typename T, bool VEC> static cudaError_t back_by_width(const NormArgs& a, int* blocks, cudaStream_t st) {
    constexpr int COLS = Chunk<T, VEC>::COLS;
    const int64_t pieces = ceil_div(a.cols, COLS);
    cudaError_t e = cudaSuccess;
    // Streams of narrow rows, a block to a wide one: in a block each warp has a piece or two, and the barrier's price is shared by few.  us, streams
    // / blocks.  60000 rows of 128 in fp32 with the residual's gradient 27 / 77; 22069 of 368 in fp32 31 / 36; 131072 of 1536 in bf16 236 / 269, with
    // the residual's gradient 327 / 295; 50000 of 2048 in bf16 with it 198 / 145; 50000 of 1000 in fp32 with it 211 / 127; 30000 of 1536 in fp32 with it
    // 224 / 131.
    if constexpr (VEC) { if (back_stream<T>(a, blocks, &e, st)) return e; }
    if (pieces <= 8) return back_go<T, VEC, 1, 4>(a, blocks, st);
    if (pieces <= 16) return back_go<T, VEC, 2, 2>(a, blocks, st);
    if (pieces <= 32) return back_go<T, VEC, 4, 1>(a, blocks, st);
    if constexpr (COLS == 128) { if (pieces <= 64) return back_go<T, VEC, 8, 1>(a, blocks, st); }
    *blocks = (int)(a.n < GEAR_NORM_WORKSPACE_ROWS ? a.n : GEAR_NORM_WORKSPACE_ROWS);
    return launch_now(rms_norm_back_wide_kernel<T>, dim3((unsigned)*blocks), dim3(256), 0, st, a);
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
    return launch_now(norm_dweight_kernel, dim3((unsigned)ceil_div(a.cols, 32)), dim3(1024), 0, st, static_cast<const float*>(a.parts), blocks,
                            a.cols, a.dweight);
}

cudaError_t launch_q8_weights(const float* W, int64_t ldw, int K, int N, uint8_t* q, int64_t ldq, float* scale, uint8_t* qt, int64_t ldqt,
                              float* scale_t, cudaStream_t st) {
    const int vec = on16(W, ldw, 4);
    const int64_t blocks = ceil_div(K, Q8_BLOCK) * ceil_div(N, Q8_BLOCK);
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;    // (weights of 2^31 blocks fit no memory)
    return launch_now(q8_weights_kernel, dim3((unsigned)blocks), dim3(QW_THREADS), 0, st, W, ldw, vec, K, N, q, ldq, scale, qt, ldqt, scale_t);
}

}  // namespace gear
