// Attention of many query columns over the 4-bit pages by the tensor cores (cf_kv4_attn where a kv head has more query columns,
// query heads times tokens, than a few; bf16 storage, head_dim 128): a follow-up question over cached documents, or the
// verification of drafted tokens.
//
// A unit is 128 query columns of a (layer, request, kv head) and the request's rows, 64 at a time.  Roles of a CTA:
//   warps 0-3   softmax, one query column per thread (= TMEM lane); its queries into tensor memory, its results out of it
//   warps 4-7   codes to fp16 keys, 16 rows each, into a swizzled shared-memory tile
//   warps 8-11  codes to fp16 values
//   warp 12     MMA issue, the warp converged and one lane elected
//   warp 13     copies of the pool's blocks
// S = Q K^T with the queries as the A operand in tensor memory, O += P V with P as the A operand over the S columns already
// consumed; two S buffers, so that S of the next tile is computed while the softmax is at this one.
// Numbers: a code times its scale is ten bits, exact in fp16 as long as the scales of a block of 16 rows lie within 2^28 of each
// other: a block is kept in units of 2^c, c chosen so that its largest scale comes to lie in [2^12, 2^13) (smaller ones lose last
// bits, 2^-38 of the block's largest number and less).  Keys' units go into the logits' factor, which is the same for the 16
// logits of a block; values' units into the probabilities, relative to the unit of O.  Queries are scaled by a power of two
// per row.  Probabilities are fp16 (11 bits), sums fp32.  O is rescaled, by the softmax warps in tensor memory, only when a
// logit lies 2^8 above the running maximum or a block's unit above that of O.
// What bounds it: see the measurements at launch_kv4_attn_tc.
#include <math_constants.h>

#include "cf_kv4_attn.cuh"
#include "cf_tc_util.cuh"

namespace cf {

using namespace kv4;

namespace {

using namespace tc;

constexpr int kRaw = 3;                           // tiles of raw blocks
constexpr int kKeys = 1 << kTcStepLog2, kBlocks = kKeys / kBlockRows;
constexpr int kKeyHalf = kKeys * 128, kKeyTile = 2 * kKeyHalf;     // bytes: 64 dims of a tile, a tile
constexpr int kBlockBytes = block_bytes(kD), kRawTile = kBlocks * kBlockBytes;
constexpr int kMmaWarp = 12, kLoadWarp = 13, kTcThreads = 448;
constexpr int kUnits = 4;                         // rings of the blocks' units (keys run three tiles ahead of the softmax) and of NaN marks
constexpr float kSlack = 8.f;
constexpr int kHead = 7;                          // P is at most 2^kSlack * 2^kHead, below fp16's 2^16
constexpr int kTmemS = 0, kTmemO = 128, kTmemQ = 256, kTmemColumns = 512;

struct TcShared {
    unsigned long long raw_full[kRaw], raw_free[kRaw], k_full[2], v_full[2], s_full[2], p_ready[2], o_done[2], q_full;
    unsigned tmem_base;
    volatile int abort_flag;
    float key_unit[kUnits][kBlocks];              // 2^c of a tile's blocks
    int value_unit[kUnits][kBlocks];              // c
    volatile int nan_unit[kUnits];                // by ordinal: that + 1 where a unit has a NaN among the values that not all of its queries see
};
constexpr int kTcSmem = 1024 + 4 * kKeyTile + kRaw * kRawTile + (int)sizeof(TcShared);

// fp16 x fp16 -> fp32, A and K-major B; B may be MN-major.
__device__ __forceinline__ uint32_t instr_desc_f16(int n, bool b_mn_major) {
    return (1u << 4) | (b_mn_major ? (1u << 16) : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTcColumns >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// A warp's block of 16 rows from codes to fp16 numbers in the swizzled tile: lane (row % 8, c) has rows row and row + 8 of dims
// 32 j + 8 c .. + 7, a 16-byte piece for each group j; the eight lanes of a store fall on all banks.  `hide`: rows from there on
// read as zeros; NaN scales in rows from `some` on too, and the answer says whether there were any.  Returns the unit's exponent.
template <bool VALUES>
__device__ __forceinline__ int expand_block(const unsigned char* raw, unsigned char* tile, int block, int hide, int some, bool& nan) {
    const int lane = threadIdx.x & 31, c = lane >> 3;
    uint32_t codes[2][4];                                    // [row half][group]
    float scale[2][4];
    float most = 0.f;
    nan = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = (lane & 7) + 8 * h;
        if (VALUES) {                                        // the two halves of a piece lie in two places, read in turn by the lanes
            const int first = 2 * c + (c & 1);
            uint2 a = *reinterpret_cast<const uint2*>(raw + value_code_at<kD>(row, first));
            uint2 b = *reinterpret_cast<const uint2*>(raw + value_code_at<kD>(row, first ^ 1));
            if (c & 1) {
                const uint2 x = a;
                a = b, b = x;
            }
            codes[h][0] = __byte_perm(a.x, b.x, 0x5410), codes[h][1] = __byte_perm(a.x, b.x, 0x7632);
            codes[h][2] = __byte_perm(a.y, b.y, 0x5410), codes[h][3] = __byte_perm(a.y, b.y, 0x7632);
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(raw + key_code_at<kD>(row) + c * (kD / 8));
            codes[h][0] = a.x, codes[h][1] = a.y, codes[h][2] = a.z, codes[h][3] = a.w;
        }
        uint2 s = *reinterpret_cast<const uint2*>(raw + (VALUES ? value_scale_at<kD>(row) : key_scale_at<kD>(row)));
        if (row >= hide) s = make_uint2(0u, 0u);
        scale[h][0] = bf16_low(s.x), scale[h][1] = bf16_high(s.x), scale[h][2] = bf16_low(s.y), scale[h][3] = bf16_high(s.y);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (VALUES && row >= some && scale[h][j] != scale[h][j]) scale[h][j] = 0.f, nan = true;
            most = fmaxf(most, scale[h][j]);
        }
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    nan = __any_sync(0xffffffffu, nan);
    const int unit = max(-110, (int)(__float_as_uint(most) >> 23) - 127 - 12);
    const float down = __int_as_float((127 - unit) << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = block * kBlockRows + (lane & 7) + 8 * h;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float s = scale[h][j] * down;
            const uint32_t s2 = pack_f16(s, s), w = codes[h][j];
            *reinterpret_cast<uint4*>(tile + (j >> 1) * kKeyHalf + swz(row, 4 * (j & 1) + c)) =
                make_uint4(mul_f16x2(two_numbers<0>(w), s2), mul_f16x2(two_numbers<1>(w), s2), mul_f16x2(two_numbers<2>(w), s2),
                           mul_f16x2(two_numbers<3>(w), s2));
        }
    }
    return unit;
}

__global__ void __launch_bounds__(kTcThreads, 1)
kv4_attn_tc_kernel(const __grid_constant__ Kv4Args args, const __grid_constant__ PagesView pv) {
    extern __shared__ unsigned char smem_raw[];
    chain_next();
    chain_wait();
    const Kv4Args& a = args;
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char *s_k = smem, *s_v = smem + 2 * kKeyTile, *s_raw = smem + 4 * kKeyTile;
    TcShared* sh = reinterpret_cast<TcShared*>(s_raw + kRaw * kRawTile);
    volatile int* abort_flag = &sh->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    asm volatile("fence.proxy.async;" ::: "memory");         // what earlier kernels wrote is read by bulk copies

    const int share = blockIdx.x, cost = a.unit_cost;
    const Line line = {pv, a.n_kv_heads * (int)a.tiles.d, cost, pv.table_cols * pv.page_rows, kTcStepLog2};
    const long long per_layer = line.length_of_layer(), total = per_layer * a.n_layers;
    const long long size = max(a.least_share, (total + a.n_shares - 1) / a.n_shares);
    const long long begin = share * size, mine = min(size, total - begin);
    if (tid == 0 && !a.marks_by_unit) a.marks[share] = make_int4(0, 0, 0, 0);
    if (share == 0 && warp == 0)
        for (int b = lane; b < pv.n_requests; b += 32)
            if (pv.rows[b] < 0 || pv.rows[b] > line.most) atomicCAS(pv.status, 0, CF_ERR_RANGE);
    if (mine <= 0) return;                                   // the whole CTA

    if (warp == kMmaWarp) {
        if (lane == 0) {
            for (int i = 0; i < kRaw; ++i) {
                mbar_init(smem_u32(&sh->raw_full[i]), kBlocks);
                mbar_init(smem_u32(&sh->raw_free[i]), 2 * kBlocks);
            }
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&sh->k_full[i]), kBlocks);
                mbar_init(smem_u32(&sh->v_full[i]), kBlocks);
                mbar_init(smem_u32(&sh->s_full[i]), 1);
                mbar_init(smem_u32(&sh->p_ready[i]), 4);
                mbar_init(smem_u32(&sh->o_done[i]), 1);
            }
            mbar_init(smem_u32(&sh->q_full), 4);
            sh->abort_flag = 0;
            for (int i = 0; i < kUnits; ++i) sh->nan_unit[i] = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "n"(kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();                                         // barriers are initialised, tensor memory is allocated
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;

    // Every warp walks the share by itself: units in order, tiles in order, `g` counts the CTA's tiles, `ordinal` its units.
    Walk p = line.find(begin, mine, per_layer);
    int g = 0, ordinal = 0;
    bool ok = true;

    if (warp == kLoadWarp) {
        // -------------------------------------------------------------- copies: lane 4 i + x looks up block x of the i-th next tile
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            const int head = a.tiles.quotient(p.unit), per_page = (int)a.blocks_per_page.d;
            for (int t0 = start; ok && t0 < last; t0 += 8) {
                const int block = (t0 + (lane >> 2)) * kBlocks + (lane & 3);
                const unsigned char* from = nullptr;
                if (t0 + (lane >> 2) < last && (block == 0 || block * kBlockRows < p.rows)) {
                    const int column = a.blocks_per_page.quotient(block);
                    int page = pv.table[(size_t)p.request * pv.table_cols + column];
                    if ((unsigned)page >= (unsigned)pv.n_pages) {
                        if (p.rows > 0) atomicCAS(pv.status, 0, CF_ERR_RANGE);
                        page = 0;
                    }
                    from = a.kv4 + (size_t)p.layer * a.kv4_layer_stride +
                           (((size_t)page * a.n_kv_heads + head) * per_page + (block - column * per_page)) * kBlockBytes;
                }
                for (int i = 0; ok && i < min(8, last - t0); ++i, ++g) {
                    const int stage = g % kRaw;
                    if (g >= kRaw) ok = warp_wait(smem_u32(&sh->raw_free[stage]), (g / kRaw - 1) & 1, abort_flag);
                    if (ok && (lane >> 2) == i) {
                        const uint32_t bar = smem_u32(&sh->raw_full[stage]);
                        if (from) {
                            mbar_expect_tx(bar, kBlockBytes);
                            bulk_load(smem_u32(s_raw + stage * kRawTile + (lane & 3) * kBlockBytes), from, kBlockBytes, bar);
                        } else {
                            mbar_arrive(bar);
                        }
                    }
                    __syncwarp();
                }
            }
        }
    } else if (warp == kMmaWarp) {
        // -------------------------------------------------------------- MMA issue
        const uint64_t dk = smem_desc(smem_u32(s_k), 16, 1024), dv = smem_desc(smem_u32(s_v), kKeyHalf, 1024);
        const uint32_t idesc_s = instr_desc_f16(kKeys, false), idesc_o = instr_desc_f16(kD, true);
        auto issue_pv = [&](int tile, bool first) {          // O (+)= P V of a tile
            const int b = tile & 1;
            ok = warp_wait(smem_u32(&sh->v_full[b]), (tile >> 1) & 1, abort_flag) && warp_wait(smem_u32(&sh->p_ready[b]), (tile >> 1) & 1, abort_flag);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kBlocks; ++kk)         // 16 keys = 8 packed P columns per instruction
                    umma_ts(tmem + kTmemO, tmem + kTmemS + b * kKeys + kk * 8, dv + (uint64_t)(b * (kKeyTile >> 4) + kk * 128), idesc_o, first && kk == 0 ? 0u : 1u);
                umma_commit(smem_u32(&sh->o_done[b]));
            }
            __syncwarp();
        };
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            ok = warp_wait(smem_u32(&sh->q_full), ordinal & 1, abort_flag);
            for (int t = start; ok && t < last; ++t, ++g) {
                const int b = g & 1;
                ok = warp_wait(smem_u32(&sh->k_full[b]), (g >> 1) & 1, abort_flag);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(tmem + kTmemS + b * kKeys, tmem + kTmemQ + kk * 8,
                                dk + (uint64_t)((b * kKeyTile + (kk >> 2) * kKeyHalf + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
                    umma_commit(smem_u32(&sh->s_full[b]));
                }
                __syncwarp();
                if (t > start) issue_pv(g - 1, t - 1 == start);
            }
            if (ok) issue_pv(g - 1, last - 1 == start);
            ++ordinal;
        }
    } else if (warp >= 4) {
        // -------------------------------------------------------------- codes to numbers
        const bool values = warp >= 8;
        const int block = warp & 3;
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            const int head = a.tiles.quotient(p.unit);
            const int all_see = p.rows - a.q_len + 1 + a.group.quotient((p.unit - head * (int)a.tiles.d) * kTcColumns);
            for (int t = start; ok && t < last; ++t, ++g) {
                const int b = g & 1, stage = g % kRaw, row0 = t * kKeys + block * kBlockRows;
                ok = warp_wait(smem_u32(&sh->raw_full[stage]), (g / kRaw) & 1, abort_flag);
                // the tile before the last in this buffer has been read
                if (ok && g >= 2) ok = warp_wait(smem_u32(values ? &sh->o_done[b] : &sh->s_full[b]), ((g >> 1) - 1) & 1, abort_flag);
                if (!ok) break;
                const unsigned char* raw = s_raw + stage * kRawTile + block * kBlockBytes;
                bool nan;
                if (values) {
                    const int unit = expand_block<true>(raw, s_v + b * kKeyTile, block, p.rows - row0, all_see - row0, nan);
                    if (lane == 0) sh->value_unit[g % kUnits][block] = unit;
                    if (nan && lane == 0) sh->nan_unit[ordinal % kUnits] = ordinal + 1;
                } else {
                    const int unit = expand_block<false>(raw, s_k + b * kKeyTile, block, p.rows - row0, 0, nan);
                    if (lane == 0) sh->key_unit[g % kUnits][block] = __int_as_float((127 + unit) << 23);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh->raw_free[stage]));
                    mbar_arrive(smem_u32(values ? &sh->v_full[b] : &sh->k_full[b]));
                }
            }
            ++ordinal;
        }
    } else {
        // -------------------------------------------------------------- softmax, one query column per thread
        const uint32_t lane_tmem = tmem + ((uint32_t)(warp * 32) << 16);
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            const int head = a.tiles.quotient(p.unit), col0 = (p.unit - head * (int)a.tiles.d) * kTcColumns, column = col0 + tid;
            const bool real = column < a.columns;
            const int token = a.group.quotient(min(column, a.columns - 1));
            const int all_see = p.rows - a.q_len + 1 + a.group.quotient(col0), sees = p.rows - a.q_len + 1 + token;
            // the queries: scaled so that the largest lies in [1, 2), two dims to a column of tensor memory
            float cs;
            {
                const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + (size_t)p.layer * a.q_layer_stride +
                                         (((size_t)p.request * a.q_len + token) * a.n_q_heads + head * (int)a.group.d + a.group.remainder(min(column, a.columns - 1))) * kD;
                uint4 w[16];
                uint32_t amax = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    w[i] = real ? *reinterpret_cast<const uint4*>(q + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t m = __vmaxu2(__vmaxu2(w[i].x & 0x7fff7fffu, w[i].y & 0x7fff7fffu), __vmaxu2(w[i].z & 0x7fff7fffu, w[i].w & 0x7fff7fffu));
                    amax = max(amax, max(m & 0xffffu, m >> 16));
                }
                int e = amax == 0 || amax >= 0x7f80u ? 0 : (int)(amax >> 7) - 127;
                e = max(-126, min(126, e));
                const float down = __int_as_float((127 - e) << 23);
                cs = a.scale_log2 * __int_as_float((127 + e) << 23);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t f[16];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint4 u = w[4 * i + x];
                        f[4 * x] = pack_f16(bf16_low(u.x) * down, bf16_high(u.x) * down), f[4 * x + 1] = pack_f16(bf16_low(u.y) * down, bf16_high(u.y) * down);
                        f[4 * x + 2] = pack_f16(bf16_low(u.z) * down, bf16_high(u.z) * down), f[4 * x + 3] = pack_f16(bf16_low(u.w) * down, bf16_high(u.w) * down);
                    }
                    tmem_st16_from<0>(lane_tmem + kTmemQ + 16 * i, f);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->q_full));
            }
            float base = 0.f, slack = -INFINITY, l = 0.f;    // as in the other kernel: the running maximum (0 before there is one), room above it
            int o_unit = 0;
            for (int t = start; ok && t < last; ++t, ++g) {
                const int b = g & 1;
                const uint32_t s_addr = lane_tmem + kTmemS + b * kKeys;
                // (not for k_full: the keys of tile g + 2 may be there before this warp looks, and a parity wait would miss the phase.  S of
                // g + 2 waits for this tile's P, and so do the values of g + 2.)
                ok = warp_wait(smem_u32(&sh->v_full[b]), (g >> 1) & 1, abort_flag) && warp_wait(smem_u32(&sh->s_full[b]), (g >> 1) & 1, abort_flag);
                if (!ok) break;
                tc_fence_after();
                float x[kBlocks][16];
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) tmem_ld16_async(s_addr + 16 * c, reinterpret_cast<uint32_t(&)[16]>(x[c]));
                float most = -INFINITY;
                int unit[kBlocks], top_unit = -1000;
                const bool masked = (t + 1) * kKeys > all_see;
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) {
                    const float f = cs * sh->key_unit[g % kUnits][c];
                    unit[c] = sh->value_unit[g % kUnits][c];
                    top_unit = max(top_unit, unit[c]);
                    tmem_ld16_wait(reinterpret_cast<uint32_t(&)[16]>(x[c]));
                    if (!masked) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[c][i] = fmaf(x[c][i], f, -base), most = fmaxf(most, x[c][i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            x[c][i] = t * kKeys + 16 * c + i < sees ? fmaf(x[c][i], f, -base) : -INFINITY;
                            most = fmaxf(most, x[c][i]);
                        }
                    }
                }
                const bool first = t == start;
                if (first) o_unit = top_unit;
                if (__any_sync(0xffffffffu, most > slack) || top_unit > o_unit) {
                    float y = most, r = 1.f;
                    if (slack != -INFINITY) y = fmaxf(y, 0.f), r = fast_exp2(-y);
                    if (y != -INFINITY) {
                        base += y, slack = kSlack;
#pragma unroll
                        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[c][i] -= y;
                    }
                    l *= r;
                    if (top_unit > o_unit) r *= exp2f((float)(o_unit - top_unit)), o_unit = top_unit;
                    if (!first) {                            // O in tensor memory, when the tile before is in it
                        ok = warp_wait(smem_u32(&sh->o_done[b ^ 1]), ((g - 1) >> 1) & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int i = 0; i < kD; i += 16) {
                            uint32_t o[16];
                            tmem_ld16_async(lane_tmem + kTmemO + i, o);
                            tmem_ld16_wait(o);
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * r);
                            tmem_st16_from<0>(lane_tmem + kTmemO + i, o);
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) {
                    const float f = exp2f((float)(kHead + unit[c] - o_unit));
                    uint32_t w[16];
                    float s0 = 0.f, s1 = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float p0 = fast_exp2(x[c][i]), p1 = fast_exp2(x[c][i + 1]);
                        s0 += p0, s1 += p1;
                        w[i >> 1] = pack_f16(p0 * f, p1 * f);
                    }
                    l += s0 + s1;
                    tmem_st8_async(s_addr + 8 * c, w);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[b]));
            }
            if (!ok) break;
            // results, or a part of them
            ok = warp_wait(smem_u32(&sh->o_done[(g - 1) & 1]), ((g - 1) >> 1) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            unsigned bad = 0;                                // groups of dims that a NaN reached
            if (sh->nan_unit[ordinal % kUnits] == ordinal + 1)
                for (int r = max(start * kKeys, max(0, all_see)); r < min(sees, last * kKeys); ++r) {
                    const int block = r / kBlockRows, col = a.blocks_per_page.quotient(block), page = pv.table[(size_t)p.request * pv.table_cols + col];
                    if ((unsigned)page >= (unsigned)pv.n_pages) continue;
                    const uint2 s = *reinterpret_cast<const uint2*>(
                        a.kv4 + (size_t)p.layer * a.kv4_layer_stride +
                        (((size_t)page * a.n_kv_heads + head) * a.blocks_per_page.d + a.blocks_per_page.remainder(block)) * kBlockBytes + value_scale_at<kD>(r % kBlockRows));
                    const float v[4] = {bf16_low(s.x), bf16_high(s.x), bf16_low(s.y), bf16_high(s.y)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) bad |= v[j] != v[j] ? 1u << j : 0u;
                }
            const bool begins = p.at <= cost, whole = begins && p.end() == p.length;
            const int slot = 2 * share + (begins ? 1 : 0);
            const float m = slack == -INFINITY ? -INFINITY : base, o_scale = exp2f((float)(o_unit - kHead));
            const float f = !whole ? o_scale : l == 0.f ? 0.f : o_scale / l;
            __nv_bfloat16* out = out_row<__nv_bfloat16, kD>(a, p.layer, p.request, head, min(column, a.columns - 1));
            float* part = a.part_o + ((size_t)slot * kTcColumns + tid) * kD;
#pragma unroll 1
            for (int i = 0; i < kD; i += 16) {
                uint32_t o[16];
                tmem_ld16_async(lane_tmem + kTmemO + i, o);
                tmem_ld16_wait(o);
                const bool nan = bad >> (i / 32) & 1;
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = nan ? 0x7fffffffu : __float_as_uint(__uint_as_float(o[j]) * f);
                if (whole) {
                    uint32_t h[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[j] = pack_bf16(__uint_as_float(o[2 * j]), __uint_as_float(o[2 * j + 1]));
                    if (real)
#pragma unroll
                        for (int j = 0; j < 8; j += 4) *reinterpret_cast<uint4*>(out + i + 2 * j) = make_uint4(h[j], h[j + 1], h[j + 2], h[j + 3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; j += 4) *reinterpret_cast<uint4*>(part + i + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                }
            }
            if (whole) {
                if (real) store_lse(a, pv.n_requests, p.layer, p.request, head, column, m, l);
            } else {
                a.part_ml[(size_t)slot * 2 * kTcColumns + tid] = m;
                a.part_ml[(size_t)slot * 2 * kTcColumns + kTcColumns + tid] = l;
            }
            if (tid == 0 && begins && (!whole || a.marks_by_unit)) {
                const long long more = p.length - p.end();
                const int lb = p.layer * pv.n_requests + p.request;
                a.marks[a.marks_by_unit ? lb * line.units + p.unit : share] = make_int4(whole ? 0 : 1 + (int)((more + size - 1) / size), share, lb, p.unit);
            }
            tc_fence_before();                               // O has been read when the next unit's queries arrive
            ++ordinal;
        }
    }

    // ---------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {
        // a wait expired: the copies in flight get the time to land before the shared memory is given back
        if (tid == 0) {
            const long long t0 = clock64();
            while (clock64() - t0 < kWaitLimitCycles / 64) {}
            atomicCAS(pv.status, 0, CF_ERR_TIMEOUT);
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColumns) : "memory");
    }
}

}  // namespace

bool kv4_attn_tc_supported(const cf_geom* g, int columns) {
#ifndef TCMIN
#define TCMIN 32
#endif
    return g->dtype == CF_BF16 && g->head_dim == kD && columns > TCMIN;
}

int launch_kv4_attn_tc(const Kv4Args& a, const PagesView& pv, cudaStream_t stream) {
    static PerDeviceOnce once;
    const int rc = configure_smem_once(once, kv4_attn_tc_kernel, kTcSmem);
    if (rc != CF_OK) return rc;
    return launch_chained(kv4_attn_tc_kernel, dim3((unsigned)a.n_shares), kTcThreads, kTcSmem, stream, a, pv);
}

}  // namespace cf
