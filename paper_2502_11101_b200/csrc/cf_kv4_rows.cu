// Rows of keys and values into the 4-bit pool and back (cf_kv4_write, cf_kv4_read).
//
// Both stream: 4 bytes in and 1.1 out per pair of numbers, or the reverse, so they are laid out for memory.  Eight lanes have a
// row of a kv head: lane u holds dims 4u .. 4u+3 of every group of 32, which are the bytes of its own value codes (8 bytes that
// lie together in the block) and half of a key word, so that one exchange with its neighbour gives each of the two 8 bytes
// of key codes to store.  A warp has four rows: together they write whole 32-byte sectors of value codes.
#include <algorithm>

#include "cf_kv4.cuh"

namespace cf {

using namespace kv4;

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowsPerWarp = 4;

__device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&x)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// A lane's four numbers of each group.  amax: the largest magnitude's upper 16 bits of groups 2i and 2i + 1, magnitudes
// ordering as integers with everything that is not finite on top; scale, codes: what a group is kept as.
template <typename T, int D> struct Numbers;

// bf16.  Quotients are needed only to tell on which side of the border between two codes they lie, and numbers of eight bits
// leave no close calls.  x / s lies on a border m / 4 (m = 1, 3, 5, 7, 10, 14, 20) exactly, or at least 2^-11 off it: x - s m / 4
// is a multiple of the smaller of x's last place and a quarter of s's, and x / s > 0.2 bounds the ratio of the two.  So x times
// an approximate 1 / s, rounded to multiples of 2^-16 (what adding 192 does), is on the border when x / s is and on the right
// side otherwise.  In the same way amax / 6 is never within 2^-11 of its size of a border between two bf16 numbers, and a
// product with 1 / 6 will do.
template <int D> struct Numbers<__nv_bfloat16, D> {
    uint2 w[D / 32];
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int u) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) w[j] = *reinterpret_cast<const uint2*>(row + 32 * j + 4 * u);
    }
    // The larger magnitude of each half, a NaN where there is one; its sign means nothing.
    __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ __forceinline__ void scales_of(uint32_t (&scales)[D / 64]) const {
        uint32_t amax[D / 64], least = 0xffffffffu, most = 0u;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint32_t a = larger(w[2 * i].x, w[2 * i].y), b = larger(w[2 * i + 1].x, w[2 * i + 1].y);
            uint32_t m = larger(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));        // of both groups
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) m = larger(m, __shfl_xor_sync(0xffffffffu, m, o));
            amax[i] = m & 0x7fff7fffu;
            const __nv_bfloat162 s = __floats2bfloat162_rn(bf16_low(amax[i]) * (1.f / 6.f), bf16_high(amax[i]) * (1.f / 6.f));
            scales[i] = *reinterpret_cast<const uint32_t*>(&s);
            least = __vminu2(least, amax[i]), most = __vmaxu2(most, amax[i]);
        }
        // scales that are not numbers above 2^-126, rare: looked at one by one
        if (__any_sync(0xffffffffu, __vminu2(least, 0x02000200u) != 0x02000200u || __vmaxu2(most, 0x7f7f7f7fu) != 0x7f7f7f7fu)) {
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                uint32_t lo = scales[i] & 0xffffu, hi = scales[i] >> 16;
                if (lo < 0x0080u) lo = 0u;
                if (hi < 0x0080u) hi = 0u;
                if ((amax[i] & 0xffffu) >= 0x7f80u) lo = 0x7fffu;
                if (amax[i] >= 0x7f800000u) hi = 0x7fffu;
                scales[i] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ uint32_t codes_of(int j, float s) const {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
        // of a group without numbers: zeros (a scale of 0 gives infinity here, a NaN itself)
        auto quotient = [&](float x) {                       // with the sign of x also where it rounds to zero
            return __uint_as_float(__float_as_uint(fmaf(x, r, 192.f) - 192.f) | (__float_as_uint(x) & 0x80000000u));
        };
        const uint32_t codes = two_codes(quotient(bf16_low(w[j].x)), quotient(bf16_high(w[j].x))) |
                               two_codes(quotient(bf16_low(w[j].y)), quotient(bf16_high(w[j].y))) << 8;
        return r < INFINITY ? codes : 0u;
    }
};

// fp32: divisions.  A quotient rounded to 24 bits is on a border (of three bits, of nine for the scale) only if the exact one
// is: the dividend's last place is more than half of the border's.
template <int D> struct Numbers<float, D> {
    float4 w[D / 32];
    __device__ __forceinline__ void load(const float* row, int u) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) w[j] = *reinterpret_cast<const float4*>(row + 32 * j + 4 * u);
    }
    __device__ __forceinline__ static uint32_t scale_of(uint32_t amax) {
        if (amax >= 0x7f800000u) return 0x7fffu;
        const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__uint_as_float(amax), 6.f)));
        return s < 1.1754944e-38f ? 0u : __float_as_uint(s) >> 16;
    }
    __device__ __forceinline__ void scales_of(uint32_t (&scales)[D / 64]) const {
        uint32_t amax[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            constexpr uint32_t kMagnitude = 0x7fffffffu;
            amax[j] = max(max(__float_as_uint(w[j].x) & kMagnitude, __float_as_uint(w[j].y) & kMagnitude),
                          max(__float_as_uint(w[j].z) & kMagnitude, __float_as_uint(w[j].w) & kMagnitude));
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) amax[j] = max(amax[j], __shfl_xor_sync(0xffffffffu, amax[j], o));
#pragma unroll
        for (int i = 0; i < D / 64; ++i) scales[i] = scale_of(amax[2 * i]) | scale_of(amax[2 * i + 1]) << 16;
    }
    __device__ __forceinline__ uint32_t codes_of(int j, float s) const {
        if (!(s > 0.f)) return 0u;
        return two_codes(__fdiv_rn(w[j].x, s), __fdiv_rn(w[j].y, s)) | two_codes(__fdiv_rn(w[j].z, s), __fdiv_rn(w[j].w, s)) << 8;
    }
};

// A lane's dims of one row: codes of groups 2i and 2i + 1 in the halves of codes[i], the scales likewise.
template <typename T, int D>
__device__ __forceinline__ void quantise(const Numbers<T, D>& x, uint32_t (&codes)[D / 64], uint32_t (&scales)[D / 64]) {
    x.scales_of(scales);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) codes[i] = x.codes_of(2 * i, bf16_low(scales[i])) | x.codes_of(2 * i + 1, bf16_high(scales[i])) << 16;
}

template <int N> __device__ __forceinline__ void store_words(unsigned char* p, const uint32_t (&w)[N]) {
    if (N == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[N - 1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
}
template <int N> __device__ __forceinline__ void load_words(const unsigned char* p, uint32_t (&w)[N]) {
    if (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x, w[N - 1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// Words of key codes from a lane's codes and back.  Lane u holds half u & 1 of the words of every group; it stores the
// words of groups (u & 1) * D/64 and up, D/64 of them, which lie together.
template <int D> __device__ __forceinline__ void to_key_words(int u, const uint32_t (&codes)[D / 64], uint32_t (&words)[D / 64]) {
    if (D == 128) {
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, u & 1 ? codes[0] : codes[D / 64 - 1], 1);
        const uint32_t mine = u & 1 ? codes[D / 64 - 1] : codes[0];
        const uint32_t lo = u & 1 ? theirs : mine, hi = u & 1 ? mine : theirs;      // of dims 8t .. 8t+3 and 8t+4 .. 8t+7
        words[0] = __byte_perm(lo, hi, 0x5410);
        words[D / 64 - 1] = __byte_perm(lo, hi, 0x7632);
    } else {
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, codes[0], 1);
        words[0] = u & 1 ? __byte_perm(theirs, codes[0], 0x7632) : __byte_perm(codes[0], theirs, 0x5410);
    }
}
template <int D> __device__ __forceinline__ void from_key_words(int u, const uint32_t (&words)[D / 64], uint32_t (&codes)[D / 64]) {
    if (D == 128) {
        const uint32_t lo = __byte_perm(words[0], words[D / 64 - 1], 0x5410), hi = __byte_perm(words[0], words[D / 64 - 1], 0x7632);
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, u & 1 ? lo : hi, 1);
        codes[0] = u & 1 ? theirs : lo;
        codes[D / 64 - 1] = u & 1 ? hi : theirs;
    } else {
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, words[0], 1);
        codes[0] = u & 1 ? __byte_perm(theirs, words[0], 0x7632) : __byte_perm(words[0], theirs, 0x5410);
    }
}

template <typename T, int D>
__device__ __forceinline__ void dequantise(const uint32_t (&codes)[D / 64], const uint32_t (&scales)[D / 64], int u, T* row) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const uint32_t w = codes[j / 2];
        const uint32_t a = j & 1 ? two_numbers<2>(w) : two_numbers<0>(w), b = j & 1 ? two_numbers<3>(w) : two_numbers<1>(w);
        const float s = j & 1 ? bf16_high(scales[j / 2]) : bf16_low(scales[j / 2]);
        const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a)), fb = __half22float2(*reinterpret_cast<const __half2*>(&b));
        const float x[4] = {fa.x * s, fa.y * s, fb.x * s, fb.y * s};
        store4(row + 32 * j + 4 * u, x);
    }
}

struct RowArgs {
    int n_rows, n_kv_heads, page_rows, n_layers;
    long long n_slots, kv_layer_stride, row_stride, kv4_layer_stride;
    const long long* slots;
    int* status;
};

// WRITE: rows to slots; otherwise slots to rows.  A warp takes four rows of `run` heads, one after the other.
template <typename T, int D, bool WRITE>
__global__ void __launch_bounds__(kRowThreads)
rows_kernel(RowArgs args, Divisor page_rows, Divisor runs, Divisor quads, int run, T* k, T* v, unsigned char* kv4) {
    chain_next();
    chain_wait();
    const RowArgs& a = args;
    const int lane = threadIdx.x & 31, u = lane & 7;
    const int item = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);      // (layer, four rows, run of heads)
    const int rest = runs.quotient(item), first = (item - rest * (int)runs.d) * run;
    const int layer = quads.quotient(rest), quad = rest - layer * (int)quads.d;
    if (layer >= a.n_layers) return;                                            // whole warps
    const int row = quad * kRowsPerWarp + (lane >> 3);
    const long long slot = row < a.n_rows ? a.slots[row] : -1;
    const bool valid = slot >= 0 && slot < a.n_slots;
    if (slot >= a.n_slots && layer == 0 && first == 0 && u == 0) atomicCAS(a.status, 0, CF_ERR_RANGE);
    if (__all_sync(0xffffffffu, !valid)) return;
    size_t at = (size_t)layer * a.kv4_layer_stride;
    int r = 0;
    constexpr int kUnroll = WRITE ? 1 : 2;
    const int per_page = a.page_rows / kBlockRows;
    if (valid) {
        const long long page = slot < 0x7fffffffLL - a.page_rows ? page_rows.quotient((int)slot) : slot / a.page_rows;
        const int in_page = (int)(slot - page * a.page_rows);
        r = in_page % kBlockRows;
        at += ((size_t)(page * a.n_kv_heads + first) * per_page + in_page / kBlockRows) * block_bytes(D);
    }
    unsigned char* block = kv4 + at;
    size_t src = (size_t)layer * a.kv_layer_stride + (size_t)(valid ? row : quad * kRowsPerWarp) * a.row_stride + first * D;
    const int n = min(run, a.n_kv_heads - first);
    const int key_code = key_code_at<D>(r) + (u >> 1) * (D / 8) + (u & 1) * (D / 16), value_code = value_code_at<D>(r, u);
#pragma unroll kUnroll
    for (int i = 0; i < n; ++i, block += (size_t)per_page * block_bytes(D), src += D) {
        uint32_t codes[D / 64], scales[D / 64], words[D / 64];
        if (WRITE) {
            Numbers<T, D> nk, nv;
            nk.load(k + src, u);
            nv.load(v + src, u);
            quantise<T, D>(nk, codes, scales);
            to_key_words<D>(u, codes, words);
            if (valid) {
                store_words<D / 64>(block + key_code, words);
                if (u == 0) store_words<D / 64>(block + key_scale_at<D>(r), scales);
            }
            quantise<T, D>(nv, codes, scales);
            if (valid) {
                store_words<D / 64>(block + value_code, codes);
                if (u == 0) store_words<D / 64>(block + value_scale_at<D>(r), scales);
            }
        } else {
            uint32_t value_codes[D / 64], value_scales[D / 64];
            load_words<D / 64>(block + key_code, words);
            load_words<D / 64>(block + key_scale_at<D>(r), scales);
            load_words<D / 64>(block + value_code, value_codes);
            load_words<D / 64>(block + value_scale_at<D>(r), value_scales);
            from_key_words<D>(u, words, codes);
            if (valid) {
                dequantise<T, D>(codes, scales, u, k + src);
                dequantise<T, D>(value_codes, value_scales, u, v + src);
            }
        }
    }
}

template <typename T, int D, bool WRITE>
int launch_rows(const RowArgs& a, const void* k, const void* v, const void* kv4, cudaStream_t stream) {
    const int quads = a.n_rows / kRowsPerWarp + (a.n_rows % kRowsPerWarp != 0);
    const long long warps = (long long)quads * a.n_kv_heads * a.n_layers;
    // a warp finds its rows once for several heads, where that leaves every SM the warps it holds four times over (2.4 M rows of a
    // head: writing with runs of 1, 2, 4, 8, 16 heads 415, 341, 302, 293, 301 us; reading 321, 286, 269, 274, 276)
    const int run = (int)std::max(1LL, std::min({(long long)a.n_kv_heads, WRITE ? 8LL : 4LL, warps / (256LL * sm_count())}));
    const int runs = (a.n_kv_heads + run - 1) / run;
    const long long items = (long long)quads * runs * a.n_layers;
    if (items > 0x7fffffffLL - 64) return CF_ERR_INVALID_ARG;
    const unsigned blocks = (unsigned)((items + kRowThreads / 32 - 1) / (kRowThreads / 32));
    return launch_chained(rows_kernel<T, D, WRITE>, dim3(blocks), kRowThreads, 0, stream, a, Divisor(a.page_rows), Divisor(runs),
                          Divisor(quads), run, static_cast<T*>(const_cast<void*>(k)), static_cast<T*>(const_cast<void*>(v)),
                          static_cast<unsigned char*>(const_cast<void*>(kv4)));
}

template <bool WRITE>
int run_rows(const cf_geom* geom, const cf_pages* pages, int n_layers, int n_rows, const int64_t* slots, const void* k, const void* v,
             long long kv_layer_stride, long long row_stride, const void* kv4, long long kv4_layer_stride, void* stream) {
    int rc = validate(geom, nullptr);
    if (rc == CF_OK) rc = check_pages(pages);
    if (rc != CF_OK) return rc;
    if (n_layers <= 0 || n_rows < 0) return CF_ERR_INVALID_ARG;
    if (n_rows == 0) return CF_OK;
    if (!slots || !k || !v || !kv4) return CF_ERR_INVALID_ARG;
    const int esize = geom->dtype == CF_BF16 ? 2 : 4;
    const long long row_elems = (long long)geom->n_kv_heads * geom->head_dim;
    for (const void* p : {k, v, kv4})
        if (reinterpret_cast<uintptr_t>(p) % 16) return CF_ERR_INVALID_ARG;
    if (row_stride < row_elems || (row_stride * esize) % 16 || (kv_layer_stride * esize) % 16 || kv4_layer_stride % 16)
        return CF_ERR_INVALID_ARG;
    if (n_layers > 1 && (kv_layer_stride < (n_rows - 1) * row_stride + row_elems ||
                         kv4_layer_stride < (long long)cf_kv4_layer_bytes(geom, pages)))
        return CF_ERR_INVALID_ARG;
    const RowArgs a = {n_rows, geom->n_kv_heads, pages->page_rows, n_layers, (long long)pages->n_pages * pages->page_rows,
                       kv_layer_stride, row_stride, kv4_layer_stride, reinterpret_cast<const long long*>(slots), pages->status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (geom->dtype == CF_BF16)
        return geom->head_dim == 128 ? launch_rows<__nv_bfloat16, 128, WRITE>(a, k, v, kv4, s) : launch_rows<__nv_bfloat16, 64, WRITE>(a, k, v, kv4, s);
    return geom->head_dim == 128 ? launch_rows<float, 128, WRITE>(a, k, v, kv4, s) : launch_rows<float, 64, WRITE>(a, k, v, kv4, s);
}

}  // namespace

}  // namespace cf

using namespace cf;

extern "C" {

size_t cf_kv4_layer_bytes(const cf_geom* geom, const cf_pages* pages) {
    if (validate(geom, nullptr) != CF_OK || check_pages(pages) != CF_OK) return 0;
    return (size_t)pages->n_pages * geom->n_kv_heads * (pages->page_rows / kv4::kBlockRows) * kv4::block_bytes(geom->head_dim);
}

int cf_kv4_write(const cf_geom* geom, const cf_pages* pages, int32_t n_layers, int32_t n_rows, const int64_t* slots,
                 const void* k, const void* v, int64_t kv_layer_stride, int64_t row_stride, void* kv4,
                 int64_t kv4_layer_stride, void* stream) {
    return run_rows<true>(geom, pages, n_layers, n_rows, slots, k, v, kv_layer_stride, row_stride, kv4, kv4_layer_stride, stream);
}

int cf_kv4_read(const cf_geom* geom, const cf_pages* pages, int32_t n_layers, int32_t n_rows, const int64_t* slots,
                const void* kv4, int64_t kv4_layer_stride, void* k, void* v, int64_t kv_layer_stride, int64_t row_stride,
                void* stream) {
    return run_rows<false>(geom, pages, n_layers, n_rows, slots, k, v, kv_layer_stride, row_stride, kv4, kv4_layer_stride, stream);
}

}  // extern "C"
