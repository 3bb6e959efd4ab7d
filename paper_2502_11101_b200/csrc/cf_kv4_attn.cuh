// What the kernels of attention over the 4-bit pages share: their arguments, the line on which the work of a call lies, and
// where results go.
#pragma once

#include <climits>

#include "cf_kv4.cuh"

namespace cf {
namespace kv4 {

struct Kv4Args {
    const void* q;
    const unsigned char* kv4;
    void* out;
    float* lse;
    float* part_o;                                // [2 shares][columns][D]
    float* part_ml;                               // [2 shares][2][columns]
    int4* marks;                                  // for the merge, by unit or by share: parts, first share, layer * requests + request, unit
    long long q_layer_stride, kv4_layer_stride, out_layer_stride;
    int n_layers, q_len, n_q_heads, n_kv_heads, columns;                   // columns = query heads of a kv head * q_len
    Divisor group, tiles, blocks_per_page;
    int n_shares, warps_per_share, unit_cost;
    int marks_by_unit;                            // a mark for every unit, where there are fewer units than shares
    Divisor cluster, units_of, requests;          // of short caches: CTAs of a unit (0: shares of the line); units of a (layer, request)
    long long least_share;
    float scale_log2;
    int no_copies;                                // nothing is copied, so that every wait runs out (cf_debug_kv4_attn)
    int wait_limit;                               // of a wait, in cycles
};

// What a call runs once costs more than its cycles: its instructions come from memory.  So no divisions of 64 bits where 32 do, and
// no functions of the library where one instruction does (one request of 1000 rows, 12/2 heads: 7.1 -> 6.3 us by exponentials alone).
__device__ __forceinline__ long long quotient_up(long long n, long long d) {
    return n + d <= INT_MAX ? (long long)(((unsigned)n + (unsigned)d - 1u) / (unsigned)d) : (n + d - 1) / d;
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((127 + e) << 23); }      // -126 <= e <= 127

// Steps of 1 << log2 keys that a request has; one without rows has one too, which writes its zeros.
__device__ __forceinline__ int steps_of(int rows, int log2) { return max(1, (rows + (1 << log2) - 1) >> log2); }

// A share's way along the line.  A unit is as long as its steps and what a unit costs besides, `cost` of them, which come first: so
// that shares over many short units are not the last to end.
struct Walk {
    int layer, request, unit;                     // unit = kv head * tiles + tile, within (layer, request)
    int rows, length;                             // rows of the request, length of the unit
    int at;                                       // place in the unit
    long long left;                               // of the share, from there on
    __device__ __forceinline__ int end() const { return (int)min((long long)length, at + left); }
    __device__ __forceinline__ int first_step(int cost) const { return max(0, at - cost); }
    __device__ __forceinline__ int last_step(int cost) const { return max(0, end() - cost); }
};

struct Line {
    const PagesView& pv;
    int units, cost;                              // units per (layer, request)
    int most;                                     // rows the table has room for
    int step_log2;
    __device__ __forceinline__ int rows_of(int b) const { return min(max(pv.rows[b], 0), most); }
    __device__ __forceinline__ long long length_of_layer() const {
        long long sum = 0;
#pragma unroll 4
        for (int b = threadIdx.x & 31; b < pv.n_requests; b += 32) sum += steps_of(rows_of(b), step_log2) + cost;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        return sum * units;
    }
    __device__ __forceinline__ Walk find(long long at, long long left, long long per_layer) const {
        const int lane = threadIdx.x & 31;
        Walk p = {};
        p.left = left;
        if (at >= per_layer) p.layer = at <= INT_MAX ? (int)at / (int)per_layer : (int)(at / per_layer), at -= p.layer * per_layer;
        for (int b0 = 0;; b0 += 32) {
            const int b = b0 + lane, rows = b < pv.n_requests ? rows_of(b) : 0, length = b < pv.n_requests ? steps_of(rows, step_log2) + cost : 0;
            long long end = (long long)length * units;
            const long long mine = end;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, end, o);
                if (lane >= o) end += x;
            }
            const unsigned behind = __ballot_sync(0xffffffffu, end > at);
            if (behind != 0 || b0 + 32 >= pv.n_requests) {
                const int src = behind != 0 ? __ffs(behind) - 1 : 0;
                p.request = b0 + src;
                p.rows = __shfl_sync(0xffffffffu, rows, src);
                p.length = __shfl_sync(0xffffffffu, length, src);
                const int within = (int)(at - __shfl_sync(0xffffffffu, end - mine, src));    // the host has seen to 32 bits
                p.unit = within / p.length;
                p.at = within - p.unit * p.length;
                return p;
            }
            at -= __shfl_sync(0xffffffffu, end, 31);
        }
    }
    // To the beginning of the next unit; there is one where something is left.
    __device__ __forceinline__ void next_unit(Walk& p) const {
        p.left -= p.end() - p.at;
        p.at = 0;
        if (p.left <= 0 || ++p.unit < units) return;
        p.unit = 0;
        if (++p.request == pv.n_requests) p.request = 0, ++p.layer;
        p.rows = rows_of(p.request);
        p.length = steps_of(p.rows, step_log2) + cost;
    }
};

template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d);
template <>
__device__ __forceinline__ void store4<float>(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* p, float a, float b, float c, float d) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}

// Results of a column: where they go, by the column's number within the kv head (token-major).
template <typename T, int D>
__device__ __forceinline__ T* out_row(const Kv4Args& a, int layer, int request, int head, int column) {
    const int token = a.group.quotient(column), h = head * (int)a.group.d + a.group.remainder(column);
    return static_cast<T*>(a.out) + (size_t)layer * a.out_layer_stride + (((size_t)request * a.q_len + token) * a.n_q_heads + h) * D;
}
__device__ __forceinline__ void store_lse(const Kv4Args& a, int n_requests, int layer, int request, int head, int column, float m, float l) {
    if (!a.lse) return;
    const int token = a.group.quotient(column), h = head * (int)a.group.d + a.group.remainder(column);
    a.lse[(((size_t)layer * n_requests + request) * a.n_q_heads + h) * a.q_len + token] = l > 0.f || l != l ? m * kLn2 + logf(l) : -INFINITY;
}

}  // namespace kv4

// The tensor-core kernel (cf_kv4_attn_tc.cu): units of kTcColumns query columns, steps of 1 << kTcStepLog2 keys, a CTA per share.
constexpr int kTcColumns = 128, kTcStepLog2 = 6;
bool kv4_attn_tc_supported(const cf_geom* g, int columns, double units);
int launch_kv4_attn_tc(const kv4::Kv4Args& a, const PagesView& pv, cudaStream_t stream);

}  // namespace cf
