// Attention of many query columns over the 4-bit pages by the tensor cores (cf_kv4_attn with more than 56 query columns of a kv head,
// query heads times tokens, and eight units; bf16 storage, head_dim 128): a follow-up question over cached documents, or the
// verification of drafted tokens.
//
// A unit is 128 query columns of a (layer, request, kv head) and the request's rows, 64 at a time.  Roles of a CTA:
//   warps 0-7   softmax, one query column per thread (= TMEM lane), two groups of four warps on tiles in turn; the queries into
//               tensor memory, the results out of it, half of the dims each
//   warps 8-11  codes to fp16 keys, 16 rows each, into a swizzled shared-memory tile
//   warps 12-15 codes to fp16 values
//   warp 16     MMA issue, the warp converged and one lane elected
//   warp 17     copies of the pool's blocks
// S = Q K^T with the queries as the A operand in tensor memory, O += P V with P as the A operand, there too; four S buffers and two
// of P, so that QK^T runs two tiles ahead and neither group waits for it.  A group reads its tile's S twice, for the maximum and
// for the probabilities; what probabilities are taken from (`base`) goes from tile to tile, so a group has to wait for the other's
// maximum, not for its probabilities.  (One group with two S buffers 52 us, two threads to a column 51, two CTAs of one group per SM
// 58, where two groups took 49; this one: see launch_kv4_attn_tc.)
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
constexpr int kTiles = 4;                         // of keys and of values
constexpr int kAhead = 2;                         // tiles that QK^T runs ahead of PV
constexpr int kKeyWarp = 8, kValueWarp = 12, kMmaWarp = 16, kLoadWarp = 17, kTcThreads = 576;
constexpr int kUnits = 8;                         // rings of what goes with a tile (keys run four tiles ahead of the softmax), and of NaN marks
constexpr float kSlack = 8.f;
constexpr int kHead = 7;                          // P is at most 2^kSlack * 2^kHead, below fp16's 2^16
constexpr int kTmemS = 0, kTmemO = 256, kTmemQ = 384, kTmemP = 448, kTmemColumns = 512;   // four S buffers, two of P

struct TcShared {
    unsigned long long raw_full[kRaw], raw_free[kRaw], full[kTiles], k_free[kTiles], v_free[kTiles], s_full[4], p_ready[2], o_done[2], q_full;
    unsigned long long based[4], exchanged[4];    // by 32 query columns: the base of a tile is known; what the groups tell each other at the end
    unsigned tmem_base;
    volatile int abort_flag;
    int wait_limit;
    float key_unit[kUnits][kBlocks];              // 2^c of a tile's blocks
    int value_unit[kUnits][kBlocks];              // c
    int o_unit[2][4];                             // of O, by the last tiles of the two groups and, as `based`, by 32 query columns
    float base[2][kTcColumns];                    // of the last tiles of the two groups; -infinity: no key seen yet
    float row[2][2][kTcColumns];                  // by parity of the exchange and group
    volatile int nan_unit[kUnits];                // by ordinal: that + 1 where a unit has a NaN among the values that not all of its queries see
};
constexpr int kTcSmem = 1024 + 2 * kTiles * kKeyTile + kRaw * kRawTile + (int)sizeof(TcShared);

// A bounded wait of a whole warp, the same answer in every lane: what a turn gives may differ from lane to lane, so the lanes vote
// on it.  There are a hundred turns for each tile among eighteen warps: the clock and the abort flag are looked at once in
// kWaitTurns of them (in every turn, waiting took two fifths of the issue slots), and turns after the first are not inlined (where
// they are 47.0 us, see launch_kv4_attn_tc).
constexpr int kWaitTurns = 256;
__device__ __noinline__ bool role_wait_on(uint32_t bar, uint32_t parity, TcShared* sh) {
    const long long t0 = clock64();
    while (true) {
#pragma unroll 1
        for (int n = 0; n < kWaitTurns; ++n)
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if (__any_sync(0xffffffffu, sh->abort_flag != 0 || clock64() - t0 > sh->wait_limit)) {
            sh->abort_flag = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool role_wait(uint32_t bar, uint32_t parity, TcShared* sh) {
    return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || role_wait_on(bar, parity, sh);
}
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

// The largest logit of a tile, of its first `valid` keys: a maximum per block, by 2 and 2, and the factor of the block's unit.
template <bool MASKED>
__device__ __forceinline__ float largest_logit(uint32_t s_addr, const float* key_unit, float cs, int valid) {
    float most = -INFINITY;
#pragma unroll
    for (int c = 0; c < kBlocks; c += 2) {
        uint32_t x[2][16];
        tmem_ld16_async(s_addr + 16 * c, x[0]);
        tmem_ld16_async(s_addr + 16 * c + 16, x[1]);
        tmem_ld16_wait(x[0]);
        tmem_ld16_wait(x[1]);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = MASKED && 16 * (c + d) + i >= valid ? -INFINITY : __uint_as_float(x[d][i]);
#pragma unroll
            for (int n = 8; n > 0; n >>= 1)
#pragma unroll
                for (int i = 0; i < n; ++i) y[i] = fmaxf(y[i], y[i + n]);
            most = fmaxf(most, y[0] * (cs * key_unit[c + d]));
        }
    }
    return most;
}

// The probabilities of a tile, its first `valid` keys, and their sum.  P is 2^lift times the probabilities of a block; below
// kLeastLift (a block whose values vanish beside others) that is not in the exponent: the sum of the probabilities is taken before.
constexpr int kLeastLift = -60;
template <bool PLAIN>
__device__ __forceinline__ void write_p(uint32_t s_addr, uint32_t p_addr, const float* key_unit, const int* value_unit, float cs, float reference, int o_unit,
                                        int valid, float& l) {
    uint32_t x[2][16];
    tmem_ld16_async(s_addr, x[0]);
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        uint32_t (&y)[16] = x[c & 1];
        tmem_ld16_wait(y);
        if (c + 1 < kBlocks) tmem_ld16_async(s_addr + 16 * (c + 1), x[(c + 1) & 1]);
        const int e = kHead + value_unit[c] - o_unit;
        const float lift = !PLAIN && e < kLeastLift ? 0.f : (float)e, f = cs * key_unit[c], add = lift - reference;
        const uint64_t f2 = pack_f2(f, f), add2 = pack_f2(add, add);
        uint64_t sum2 = 0;
        if (PLAIN) {
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float p0, p1;
                unpack_f2(fma_f2(pack_f2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), f2, add2), p0, p1);
                p0 = fast_exp2(p0), p1 = fast_exp2(p1);
                sum2 = add_f2(sum2, pack_f2(p0, p1));
                y[i >> 1] = pack_f16(p0, p1);
            }
        } else {
            const float after = e < kLeastLift ? exp2f((float)e) : 1.f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float p0 = 16 * c + i < valid ? fast_exp2(fmaf(__uint_as_float(y[i]), f, add)) : 0.f;
                const float p1 = 16 * c + i + 1 < valid ? fast_exp2(fmaf(__uint_as_float(y[i + 1]), f, add)) : 0.f;
                sum2 = add_f2(sum2, pack_f2(p0, p1));
                y[i >> 1] = pack_f16(p0 * after, p1 * after);
            }
        }
        float s0, s1;
        unpack_f2(sum2, s0, s1);
        l = fmaf(s0 + s1, __int_as_float((127 - (int)lift) << 23), l);
        tmem_st8_async(p_addr + 8 * c, y);
    }
}

__global__ void __launch_bounds__(kTcThreads, 1)
kv4_attn_tc_kernel(const __grid_constant__ Kv4Args args, const __grid_constant__ PagesView pv) {
    extern __shared__ unsigned char smem_raw[];
    chain_next();
    chain_wait();
    const Kv4Args& a = args;
    unsigned char* smem = smem_raw + (-smem_u32(smem_raw) & 1023u);
    unsigned char *s_k = smem, *s_v = smem + kTiles * kKeyTile, *s_raw = smem + 2 * kTiles * kKeyTile;
    TcShared* sh = reinterpret_cast<TcShared*>(s_raw + kRaw * kRawTile);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    asm volatile("fence.proxy.async;" ::: "memory");         // what earlier kernels wrote is read by bulk copies

    const int share = blockIdx.x, cost = a.unit_cost;
    const Line line = {pv, a.n_kv_heads * (int)a.tiles.d, cost, pv.table_cols * pv.page_rows, kTcStepLog2};
    const long long per_layer = line.length_of_layer(), total = per_layer * a.n_layers;
    const long long size = max(a.least_share, quotient_up(total, a.n_shares));
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
            for (int i = 0; i < kTiles; ++i) {
                mbar_init(smem_u32(&sh->full[i]), 2 * kBlocks);
                mbar_init(smem_u32(&sh->k_free[i]), 1);
                mbar_init(smem_u32(&sh->v_free[i]), 1);
            }
            for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&sh->s_full[i]), 1);
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&sh->p_ready[i]), 4);
                mbar_init(smem_u32(&sh->o_done[i]), 1);
            }
            for (int i = 0; i < 4; ++i) {
                mbar_init(smem_u32(&sh->based[i]), 1);
                mbar_init(smem_u32(&sh->exchanged[i]), 2);
            }
            mbar_init(smem_u32(&sh->q_full), 8);
            sh->abort_flag = 0, sh->wait_limit = a.wait_limit;
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
                    if (g >= kRaw) ok = role_wait(smem_u32(&sh->raw_free[stage]), (g / kRaw - 1) & 1, sh);
                    if (ok && (lane >> 2) == i && !a.no_copies) {
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
            const int b = tile & 1, v = tile % kTiles;
            ok = role_wait(smem_u32(&sh->p_ready[b]), (tile >> 1) & 1, sh);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kBlocks; ++kk)         // 16 keys = 8 packed P columns per instruction
                    umma_ts(tmem + kTmemO, tmem + kTmemP + b * (kKeys / 2) + kk * 8, dv + (uint64_t)(v * (kKeyTile >> 4) + kk * 128), idesc_o, first && kk == 0 ? 0u : 1u);
                umma_commit(smem_u32(&sh->o_done[b]));
                umma_commit(smem_u32(&sh->v_free[v]));
            }
            __syncwarp();
        };
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            ok = role_wait(smem_u32(&sh->q_full), ordinal & 1, sh);
            for (int t = start; ok && t < last + kAhead; ++t) {
                if (t < last) {
                    const int k = g % kTiles;
                    // the values too: with S the softmax has the units of both
                    ok = role_wait(smem_u32(&sh->full[k]), (g / kTiles) & 1, sh);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {                       // over S of the tile four before, whose P has been waited for
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
                            umma_ts(tmem + kTmemS + (g & 3) * kKeys, tmem + kTmemQ + kk * 8,
                                    dk + (uint64_t)((k * kKeyTile + (kk >> 2) * kKeyHalf + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
                        umma_commit(smem_u32(&sh->s_full[g & 3]));
                        umma_commit(smem_u32(&sh->k_free[k]));
                    }
                    __syncwarp();
                    ++g;
                }
                if (t - kAhead >= start) issue_pv(g - (min(t + 1, last) - (t - kAhead)), t - kAhead == start);
            }
            ++ordinal;
        }
    } else if (warp >= kKeyWarp) {
        // -------------------------------------------------------------- codes to numbers
        const bool values = warp >= kValueWarp;
        const int block = warp & 3;
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            const int head = a.tiles.quotient(p.unit);
            const int all_see = p.rows - a.q_len + 1 + a.group.quotient((p.unit - head * (int)a.tiles.d) * kTcColumns);
            for (int t = start; ok && t < last; ++t, ++g) {
                const int k = g % kTiles, stage = g % kRaw, row0 = t * kKeys + block * kBlockRows;
                ok = role_wait(smem_u32(&sh->raw_full[stage]), (g / kRaw) & 1, sh);
                // the tile that was in this buffer has been read
                if (ok && g >= kTiles) ok = role_wait(smem_u32(values ? &sh->v_free[k] : &sh->k_free[k]), (g / kTiles - 1) & 1, sh);
                if (!ok) break;
                const unsigned char* raw = s_raw + stage * kRawTile + block * kBlockBytes;
                bool nan;
                if (values) {
                    const int unit = expand_block<true>(raw, s_v + k * kKeyTile, block, p.rows - row0, all_see - row0, nan);
                    if (lane == 0) sh->value_unit[g % kUnits][block] = unit;
                    if (nan && lane == 0) sh->nan_unit[ordinal % kUnits] = ordinal + 1;
                } else {
                    const int unit = expand_block<false>(raw, s_k + k * kKeyTile, block, p.rows - row0, 0, nan);
                    if (lane == 0) sh->key_unit[g % kUnits][block] = __int_as_float((127 + unit) << 23);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh->raw_free[stage]));
                    mbar_arrive(smem_u32(&sh->full[k]));
                }
            }
            ++ordinal;
        }
    } else {
        // -------------------------------------------------------------- softmax, one query column per thread, tiles in turn
        const int group = warp >> 2, quad = warp & 3, r = tid & (kTcColumns - 1);
        const uint32_t lane_tmem = tmem + ((uint32_t)(quad * 32) << 16), p_addr = lane_tmem + kTmemP + group * (kKeys / 2);
        // logits rise with q . k: the sign of the scale goes into the queries
        const float scale = fabsf(a.scale_log2);
        const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;
        int exchanges = 0;
        // What the other group's thread of the column gives for `mine`.
        auto exchange = [&](float mine) {
            const int turn = exchanges++ & 1;
            sh->row[turn][group][r] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->exchanged[quad]));
            ok = role_wait(smem_u32(&sh->exchanged[quad]), turn, sh);
            return sh->row[turn][group ^ 1][r];
        };
        for (; ok && p.left > 0; line.next_unit(p)) {
            const int start = p.first_step(cost), last = p.last_step(cost);
            if (last <= start) continue;
            const int head = a.tiles.quotient(p.unit), col0 = (p.unit - head * (int)a.tiles.d) * kTcColumns, column = col0 + r;
            const bool real = column < a.columns;
            const int token = a.group.quotient(min(column, a.columns - 1));
            const int all_see = p.rows - a.q_len + 1 + a.group.quotient(col0), sees = p.rows - a.q_len + 1 + token;
            // the queries: scaled so that the largest lies in [1, 2), two dims to a column of tensor memory
            float cs;
            {
                const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + (size_t)p.layer * a.q_layer_stride +
                                         (((size_t)p.request * a.q_len + token) * a.n_q_heads + head * (int)a.group.d + a.group.remainder(min(column, a.columns - 1))) * kD;
                uint4 w[8];
                uint32_t amax = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h)                  // both halves of the dims for the maximum, this group's last, to keep
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        w[i] = real ? *reinterpret_cast<const uint4*>(q + (h == 0 ? group ^ 1 : group) * (kD / 2) + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
                        const uint32_t m = __vmaxu2(__vmaxu2(w[i].x & 0x7fff7fffu, w[i].y & 0x7fff7fffu), __vmaxu2(w[i].z & 0x7fff7fffu, w[i].w & 0x7fff7fffu));
                        amax = max(amax, max(m & 0xffffu, m >> 16));
                    }
                int e = amax == 0 || amax >= 0x7f80u ? 0 : (int)(amax >> 7) - 127;
                e = max(-126, min(126, e));
                const float down = __int_as_float((127 - e) << 23);
                cs = scale * __int_as_float((127 + e) << 23);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t f[16];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint32_t u[4] = {w[4 * i + x].x, w[4 * i + x].y, w[4 * i + x].z, w[4 * i + x].w};
#pragma unroll
                        for (int y = 0; y < 4; ++y) f[4 * x + y] = pack_f16(bf16_low(u[y]) * down, bf16_high(u[y]) * down) ^ sign;
                    }
                    tmem_st16_from<0>(lane_tmem + kTmemQ + group * (kD / 4) + 16 * i, f);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->q_full));
            }
            // what the probabilities of the group's last tile were taken from (-infinity: no key seen), and their sum
            float base = -INFINITY, l = 0.f;
            int o_unit = -1000;                              // of the tile before, in either group
            for (int t = start; t < last; ++t, ++g) {
                if ((g & 1) != group) continue;
                const int* value_unit = sh->value_unit[g % kUnits];
                const float* key_unit = sh->key_unit[g % kUnits];
                const uint32_t s_addr = lane_tmem + kTmemS + (g & 3) * kKeys;
                ok = role_wait(smem_u32(&sh->s_full[g & 3]), (g >> 2) & 1, sh);
                if (!ok) break;
                tc_fence_after();
                const bool masked = (t + 1) * kKeys > all_see;
                // the largest logit: S is read once for it and once for the probabilities
                const float most = masked ? largest_logit<true>(s_addr, key_unit, cs, sees - t * kKeys) : largest_logit<false>(s_addr, key_unit, cs, 0);
                int top_unit = value_unit[0], low_unit = value_unit[0];
#pragma unroll
                for (int c = 1; c < kBlocks; ++c) top_unit = max(top_unit, value_unit[c]), low_unit = min(low_unit, value_unit[c]);
                // the base and the unit of O of the tile before, and then of this one
                float from = -INFINITY;
                o_unit = -1000;
                if (t > start) {
                    ok = role_wait(smem_u32(&sh->based[quad]), (g - 1) & 1, sh);
                    if (!ok) break;
                    from = sh->base[group ^ 1][r];
                    o_unit = sh->o_unit[group ^ 1][quad];
                }
                float now = from;
                if (most > from + kSlack) now = most;        // also where nothing has been seen so far
                const int now_unit = max(o_unit, top_unit);
                sh->base[group][r] = now;
                if (lane == 0) sh->o_unit[group][quad] = now_unit;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->based[quad]));
                if (base != now && base != -INFINITY) l *= fast_exp2(base - now);
                base = now;
                if (t > start && __any_sync(0xffffffffu, from != now || o_unit != now_unit)) {
                    // O in tensor memory, when the tile before is in it
                    const float f = (from == now || from == -INFINITY ? 1.f : fast_exp2(from - now)) * exp2f((float)(o_unit - now_unit));
                    ok = role_wait(smem_u32(&sh->o_done[group ^ 1]), ((g - 1) >> 1) & 1, sh);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int i = 0; i < kD; i += 16) {
                        uint32_t o[16];
                        tmem_ld16_async(lane_tmem + kTmemO + i, o);
                        tmem_ld16_wait(o);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                        tmem_st16_from<0>(lane_tmem + kTmemO + i, o);
                    }
                }
                o_unit = now_unit;
                if (g >= 2) {                                // PV has read the P that the group left last
                    ok = role_wait(smem_u32(&sh->o_done[group]), ((g >> 1) - 1) & 1, sh);
                    if (!ok) break;
                    tc_fence_after();
                }
                const float reference = now == -INFINITY ? 0.f : now;
                if (!masked && kHead + low_unit - o_unit >= kLeastLift) write_p<true>(s_addr, p_addr, key_unit, value_unit, cs, reference, o_unit, kKeys, l);
                else write_p<false>(s_addr, p_addr, key_unit, value_unit, cs, reference, o_unit, sees - t * kKeys, l);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[group]));
            }
            if (!ok) break;
            // the last tile's base and unit, and the sum of both groups
            float final_base = base;
            {
                const float theirs = exchange(base), sum = ok ? exchange(l) : 0.f;
                if (!ok) break;
                const bool last_is_mine = ((g - 1) & 1) == group;
                final_base = last_is_mine ? base : theirs;
                const float mine_f = base == final_base || base == -INFINITY ? 1.f : fast_exp2(base - final_base);
                const float their_f = theirs == final_base || theirs == -INFINITY ? 1.f : fast_exp2(theirs - final_base);
                l = l * mine_f + sum * their_f;
                o_unit = sh->o_unit[(g - 1) & 1][quad];
            }
            // results, or a part of them
            ok = role_wait(smem_u32(&sh->o_done[(g - 1) & 1]), ((g - 1) >> 1) & 1, sh);
            if (!ok) break;
            tc_fence_after();
            unsigned bad = 0;                                // groups of dims that a NaN reached
            if (sh->nan_unit[ordinal % kUnits] == ordinal + 1)
                for (int row = max(start * kKeys, max(0, all_see)); row < min(sees, last * kKeys); ++row) {
                    const int block = row / kBlockRows, col = a.blocks_per_page.quotient(block), page = pv.table[(size_t)p.request * pv.table_cols + col];
                    if ((unsigned)page >= (unsigned)pv.n_pages) continue;
                    const uint2 s = *reinterpret_cast<const uint2*>(
                        a.kv4 + (size_t)p.layer * a.kv4_layer_stride +
                        (((size_t)page * a.n_kv_heads + head) * a.blocks_per_page.d + a.blocks_per_page.remainder(block)) * kBlockBytes + value_scale_at<kD>(row % kBlockRows));
                    const float v[4] = {bf16_low(s.x), bf16_high(s.x), bf16_low(s.y), bf16_high(s.y)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) bad |= v[j] != v[j] ? 1u << j : 0u;
                }
            const bool begins = p.at <= cost, whole = begins && p.end() == p.length;
            const int slot = 2 * share + (begins ? 1 : 0);
            const float m = final_base, o_scale = exp2f((float)(o_unit - kHead));
            const float f = !whole ? o_scale : l == 0.f ? 0.f : o_scale / l;
            __nv_bfloat16* out = out_row<__nv_bfloat16, kD>(a, p.layer, p.request, head, min(column, a.columns - 1));
            float* part = a.part_o + ((size_t)slot * kTcColumns + r) * kD;
#pragma unroll 1
            for (int i = group * (kD / 2); i < (group + 1) * (kD / 2); i += 16) {
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
            if (group == 0) {
                if (whole) {
                    if (real) store_lse(a, pv.n_requests, p.layer, p.request, head, column, m, l);
                } else {
                    a.part_ml[(size_t)slot * 2 * kTcColumns + r] = m;
                    a.part_ml[(size_t)slot * 2 * kTcColumns + kTcColumns + r] = l;
                }
            }
            if (tid == 0 && begins && (!whole || a.marks_by_unit)) {
                const long long more = p.length - p.end();
                const int lb = p.layer * pv.n_requests + p.request;
                a.marks[a.marks_by_unit ? lb * line.units + p.unit : share] = make_int4(whole ? 0 : 1 + (int)quotient_up(more, size), share, lb, p.unit);
            }
            tc_fence_before();                               // O has been read when the next unit's queries arrive
            ++ordinal;
        }
    }

    // ---------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {
        // A wait expired.  What the share's units leave for the join is not all there, and a mark that was not written would send it
        // anywhere: nothing is joined of the units that begin here.
        if (warp == 0) {
            for (Walk w = line.find(begin, mine, per_layer); w.left > 0; line.next_unit(w))
                if (lane == 0 && w.at <= cost && w.end() > cost)
                    a.marks[a.marks_by_unit ? (w.layer * pv.n_requests + w.request) * line.units + w.unit : share] = make_int4(0, 0, 0, 0);
        }
        // the copies in flight get the time to land before the shared memory is given back
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

// More than 56 query columns, and eight units: below, the kernel of cf_kv4_attn.cu is faster, whose units are 16 columns.  Measured
// (that one / this one, us, 48, 64 and 128 columns): 4 requests of 4-16 K rows, 32/4 heads 30.1 / 30.9, 35.4 / 31.4, 59.2 / 33.8; 32 of
// 200-2000 rows 29.8 / 35.3, 35.9 / 36.2, 61.6 / 40.0; one of 8000 rows (four units) 15.4 / 20.1, 16.4 / 20.8, 21.3 / 23.1; one of 500
// 11.4 / 16.6, 12.1 / 16.9, 12.6 / 18.6.
bool kv4_attn_tc_supported(const cf_geom* g, int columns, double units) {
    return g->dtype == CF_BF16 && g->head_dim == kD && columns > 56 && units >= 8;
}

// 24 query tokens over 4 requests of 4-16 K rows, 28/4 heads (168 columns): 45.1 us with the join of the parts, 77 by the kernel of
// cf_kv4_attn.cu; 13.7 GFLOP, 0.19 of the measured peak.  A tile of 64 keys takes 1650 cycles, of which its products are 512, at 0.53
// of the issue slots.  Where a tile took 1700 (46.6 us, with another loop that waits) a softmax group was busy for 3400 of every two
// tiles, the warps of the values for 1650 of each, the MMA warp for 1600, all with latencies (a wait for a barrier that is complete
// took 200).  So no role alone is what bounds it: from there, without the exponentials, the conversions, the maximum or half of the
// products 45.8; three groups 48.9, eight warps of values 48.5, both 49.6, five or eight tiles of raw blocks 47.0 and 47.8.
int launch_kv4_attn_tc(const Kv4Args& a, const PagesView& pv, cudaStream_t stream) {
    static PerDeviceOnce once;
    const int rc = configure_smem_once(once, kv4_attn_tc_kernel, kTcSmem);
    if (rc != CF_OK) return rc;
    return launch_chained(kv4_attn_tc_kernel, dim3((unsigned)a.n_shares), kTcThreads, kTcSmem, stream, a, pv);
}

}  // namespace cf
