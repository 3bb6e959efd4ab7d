// Attention over the paged cache held in 4 bits (cf_kv4_attn).
//
//   out = sum_i p_i v_i / sum_i p_i,  p_i = 2^(x_i - m),  x_i = (q . k_i) * scale * log2(e),  k_i = s_k[i][j] c_k,  v_i = s_v[i][j] c_v
// with one scale s per group j of 32 dims and codes c of 4 bits, 4.5 bits per number: a quarter of the bytes of a bf16 cache, and
// 2 to 60 flops per byte, so the pass is bound by HBM as long as turning codes into matrix operands costs little.
//   S^T = K Q^T   m16n8k16, rows = 16 keys, columns = 8 queries.  The codes go into the products as they are (fp16 holds
//                 them exactly; the conversion gives two numbers an instruction); each group's partial sums are
//                 multiplied by its scale in fp32, four multiply-adds per lane and group.  Queries are scaled by a power of two
//                 per row so that bf16 fits fp16: the products are exact.
//   O^T += V^T P^T  rows = dims, columns = queries, contraction over the keys.  The values' scales go into the
//                 probabilities, one set per group: P_j = p * s_v[.][j] in fp32, rounded to fp16 (11 bits), under a power of two
//                 that follows the largest scale seen, and transposed between the lanes by movmatrix.  Codes of two keys are
//                 paired by bit operations, so that one conversion gives a register of the fragment.
// Storage in fp32 splits queries and probabilities into two fp16 numbers each (22 bits) and issues every product twice.
// The running maximum is raised only when a logit lies more than 2^8 above it: fp16 has room for that, and the
// test is one vote of the warp.
//
// A step is two blocks of 16 rows (4608 bytes at head_dim 128), one bulk copy into a ring of two steps that belongs to the
// warp: no barrier between warps, and up to 147 KB in flight per SM.  The steps of all units (layer, request, kv head, tile of query columns)
// lie end to end on one line, which is cut into equal shares; lengths are device data, so every warp finds its place by
// walking the requests' lengths.  A share belongs to a warp where there are many units, else to the warps of a CTA, which
// take its steps in turn and join their results in shared memory.  Units cut between shares leave parts in the workspace, which
// kv4_merge_kernel joins.
//
// Short caches do without the line: a unit has a cluster of CTAs, joined over distributed shared memory (see cut_of).
//
// Measured (B200, a call with its merge, caches in HBM): 8 requests of 19-21.6 K rows, 32/32 heads, 137 us call after call (5.5 TB/s,
// 0.84 of the copy rate; 122 to 127 in a cool part); 96 of 17-6001 rows, 28/4, 44.5 us (3.7 TB/s); four layers of three ragged
// requests, 32/8, 16.2 us; one of 1011 rows, 12/2, in a table with room for 1152, 6.2 us.  The loop issues 222 (few columns) and 282
// instructions for 16 keys, 64 of them conversions, at 0.57 and 0.52 per cycle and scheduler.  Few columns meet HBM; grouped heads have
// three warps to a scheduler, whose instructions and the latencies that they do not hide for one another bound them by halves.
// What the steps of its making gave (8 long 32/32 / 96 of 28/4, us): 16 keys a step, selects under masks 171 / 69; those behind a
// branch 162 / 68; 32 keys, shares weighed by units 148 / 51; a column per (query, group) 122 / -; four warps a CTA with 168
// registers - / 47; shares of single warps - / 45.
#include <algorithm>
#include <climits>

#include "cf_kv4_attn.cuh"
#include "cf_tc_util.cuh"

namespace cf {

using namespace kv4;
using tc::mbar_init;
using tc::mbar_expect_tx;
using tc::smem_u32;

namespace {

constexpr int kStages = 2;                        // steps of the ring
constexpr int kStepBlocks = 2;                    // blocks of a step
constexpr int kStepLog2 = 5, kStepRows = kStepBlocks * kBlockRows;
static_assert(kStepRows == 1 << kStepLog2, "a step's keys");
constexpr int kMergeThreads = 256;
constexpr float kSlack = 8.f;                     // how far a logit may lie above the running maximum (base 2)
constexpr int kHead = 7;                          // P is at most 2^kSlack * 2^kHead, below fp16's 2^16
constexpr int kLeastExponent = -110;
constexpr int kMostCost = 32;                     // of a unit, in steps
// A share is at least this long, in steps; a unit costs this much besides its steps (its queries, the join of its parts); by
// the warps that have a share of their own, or the CTA that has one.
constexpr int kLeastAlone = 4, kLeastTogether = 8;
constexpr int kCostAlone = 3, kCostTogether = 16;
constexpr int kMostCluster = 8;
constexpr int kClusterSteps = 6, kClusterStepsFew = 9;     // a warp has fewer steps than this where a cluster has a unit; with few columns
constexpr int kLeastTc = 8, kCostTc = 6;          // of the tensor-core kernel, in steps of its own

// Warps of a CTA, and CTAs of an SM.  With few columns the loop fits 128 registers: 16 warps per SM; without, and with twice the
// columns, fewer warps with more registers are faster.
__host__ __device__ constexpr int warps_of(bool few) { return few ? 8 : 4; }
__host__ __device__ constexpr int ctas_per_sm(int nt, bool few) { return few ? 2 : nt == 1 ? 3 : 2; }

// Query columns of a unit.
__host__ __device__ constexpr int tile_columns(int head_dim, int nt, bool few) { return few ? 8 / (head_dim / 32) : 8 * nt; }

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// What fp16 leaves of lo and hi.
__device__ __forceinline__ uint32_t pack_f16_rest(float lo, float hi, uint32_t packed) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
    return pack_f16(lo - f.x, hi - f.y);
}
// Sixteen bytes, and four, of the shared memory of another CTA of the cluster, at the place that `p` has in this one's.
__device__ __forceinline__ float4 cluster_load4(const float* p, int rank) {
    float4 x;
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %4, %5;\nld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}"
                 : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(smem_u32(p)), "r"(rank) : "memory");
    return x;
}
__device__ __forceinline__ float cluster_load(const float* p, int rank) {
    float x;
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %1, %2;\nld.shared::cluster.f32 %0, [a];\n}" : "=f"(x) : "r"(smem_u32(p)), "r"(rank) : "memory");
    return x;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(a));
    return x;
}
template <int N> __device__ __forceinline__ void lds(uint32_t a, uint32_t (&w)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "words of one load");
    if constexpr (N == 1) w[0] = lds32(a);
    if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a));
    if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
}

// The copies of a warp's steps: it takes every stride-th step from `first` on of each unit of its share.  The walk lies in shared
// memory: it is looked at once in 32 steps.
template <int D>
struct Feeder {
    static constexpr int kBytes = block_bytes(D);
    static constexpr int kNone = INT_MIN;         // no distance: a pool of 2^31 blocks has over 2 TB
    const PagesView& pv;
    const Kv4Args& a;
    const Line& line;
    Walk* walk;
    int* next;                                    // the unit's next step to look up
    int first, stride, lane;
    int ready, used;                              // steps that the lanes have looked up, one each; how many of them were issued
    const unsigned char* address;                 // a lane's step: its first block,
    int second;                                   // and how many blocks behind that its second one lies (in the same one, 0, where a
                                                  // table names a page of 16 rows twice in a row), kNone where it has none
    uint32_t ring, bars;
    unsigned issued;
    bool ended;

    __device__ __forceinline__ int page_of(int request, int rows, int column) const {
        const int page = pv.table[(size_t)request * pv.table_cols + column];
        if ((unsigned)page < (unsigned)pv.n_pages) return page;
        if (rows > 0) atomicCAS(pv.status, 0, CF_ERR_RANGE);       // a request without rows has no pages
        return 0;
    }
    __device__ __forceinline__ void look_up() {
        __syncwarp();
        Walk p = *walk;
        int step = *next;
        __syncwarp();
        ready = used = 0;
        while (p.left > 0 && !a.no_copies) {
            const int last = p.last_step(line.cost);
            const int n = step < last ? (last - step + stride - 1) / stride : 0;
            if (n > 0) {
                ready = min(32, n);
                if (lane < ready) {
                    const int per_page = (int)a.blocks_per_page.d, block = kStepBlocks * (step + lane * stride);
                    const int column = a.blocks_per_page.quotient(block), in_page = block - column * per_page;
                    const int head = a.tiles.quotient(p.unit), page = page_of(p.request, p.rows, column);
                    address = a.kv4 + (size_t)p.layer * a.kv4_layer_stride + (((size_t)page * a.n_kv_heads + head) * per_page + in_page) * kBytes;
                    second = (block + 1) * kBlockRows >= p.rows ? kNone : 1;
                    if (second != kNone && in_page + 1 == per_page)
                        second = (page_of(p.request, p.rows, column + 1) - page) * a.n_kv_heads * per_page - in_page;
                }
                step += ready * stride;
                break;
            }
            line.next_unit(p);
            step = first;
        }
        if (lane == 0) *walk = p, *next = step;
        __syncwarp();
    }
    __device__ __forceinline__ static void copy(uint32_t to, const unsigned char* from, uint32_t bytes, uint32_t bar) {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
                     : "memory");
    }
    // Issues the next step's copies into the stage that was read last.
    __device__ __forceinline__ void feed() {
        if (used == ready) {
            if (ended) return;
            look_up();
            ended = ready == 0;
            if (ended) return;
        }
        if (lane == used) {
            const uint32_t stage = issued % kStages, bar = bars + 8 * stage, to = ring + stage * kStepBlocks * kBytes;
            mbar_expect_tx(bar, second != kNone ? 2 * kBytes : kBytes);
            copy(to, address, second == 1 ? 2 * kBytes : kBytes, bar);
            if (second != kNone && second != 1) copy(to + kBytes, address + (long long)second * kBytes, kBytes, bar);
        }
        ++used;
        ++issued;
    }
};

template <typename T> struct IsF32 { static constexpr bool value = sizeof(T) == 4; };

// A part of a column's dims, or the sum of several.
struct Part {
    float top, sum;
    float4 x;
    __device__ __forceinline__ void add(float m, float l, const float4& y) {
        // without a key m is -infinity and the rest 0 (or, where it saw only NaN, NaN): times 0 or 1 that stays
        const float to = fmaxf(top, m), f0 = top == to ? 1.f : exp2_fast(top - to), f1 = m == to ? 1.f : exp2_fast(m - to);
        sum = fmaf(sum, f0, l * f1);
        x.x = fmaf(x.x, f0, y.x * f1), x.y = fmaf(x.y, f0, y.y * f1), x.z = fmaf(x.z, f0, y.z * f1), x.w = fmaf(x.w, f0, y.w * f1);
        top = to;
    }
};

// FEW: the query columns times the groups fit the eight columns of a matrix product, which then has a column per (query, group):
// one chain of products for all groups, and one set of probabilities instead of one per group.
template <typename T, int D, int NT, bool FEW>
__global__ void __launch_bounds__(32 * warps_of(FEW), ctas_per_sm(NT, FEW))
kv4_attn_kernel(Kv4Args args, PagesView pv) {
    chain_next();
    constexpr int kWarps = warps_of(FEW), kThreads = 32 * kWarps;
    constexpr int kBytes = block_bytes(D);
    constexpr int kRing = kStages * kStepBlocks * kBytes;    // of a warp
    constexpr int kGroups = D / 32;
    constexpr int kCols = tile_columns(D, NT, FEW);          // query columns of a unit
    constexpr int kOwn = FEW ? 1 : 2 * NT;                   // of which a lane has the logits of this many
    constexpr int kScaleWords = FEW ? 1 : kGroups / 2;       // scales of a key that a lane reads, two to a word
    constexpr int kParts = IsF32<T>::value ? 2 : 1;          // fp16 numbers per query or probability
    constexpr int kOStride = D + 4;                          // floats between columns in shared memory: no bank conflicts
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* s_ring = smem;                            // [kWarps][kRing]
    float* s_o = reinterpret_cast<float*>(smem + kWarps * kRing);               // [kWarps][kCols][kOStride]
    float* s_m = s_o + kWarps * kCols * kOStride;            // [kWarps][kCols]
    float* s_l = s_m + kWarps * kCols;                       // [kWarps][kCols]
    unsigned long long* s_bars = reinterpret_cast<unsigned long long*>(s_l + kWarps * kCols);   // [kWarps][kStages]
    float* s_part = reinterpret_cast<float*>(smem);          // over the ring, of a unit that a cluster shares: [kCols][D] and
    float* s_part_ml = s_part + kCols * D;                   // [2][kCols]
    __shared__ Walk s_walk[kWarps];
    __shared__ int s_next[kWarps];
    __shared__ volatile int s_abort;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    if (lane < kStages) mbar_init(smem_u32(s_bars + warp * kStages + lane), 1);
    if (tid == 0) s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    chain_wait();
    const Kv4Args& a = args;
    asm volatile("fence.proxy.async;" ::: "memory");         // what earlier kernels wrote is read by bulk copies

    const bool together = a.warps_per_share > 1;             // the CTA's warps share a share
    const int n_cluster = (int)a.cluster.d;                  // CTAs that share a unit, 0 for shares of the line
    const int share = together ? (int)blockIdx.x : (int)blockIdx.x * kWarps + warp;
    const int cost = a.unit_cost;
    const Line line = {pv, a.n_kv_heads * (int)a.tiles.d, cost, pv.table_cols * pv.page_rows, kStepLog2};
    const bool writer = lane == 0 && (!together || warp == 0);
    Walk p = {};
    long long size = 0;
    int first_step = together ? warp : 0, stride = together ? kWarps : 1, rank = 0;
    if (n_cluster > 0) {
        const int u = a.cluster.quotient((int)blockIdx.x), lb = a.units_of.quotient(u);
        rank = (int)blockIdx.x - u * n_cluster;
        first_step = rank * kWarps + warp, stride = n_cluster * kWarps;
        p.unit = u - lb * line.units;
        p.layer = a.requests.quotient(lb), p.request = lb - p.layer * pv.n_requests;
        const int rows = pv.rows[p.request];
        if ((rows < 0 || rows > line.most) && tid == 0) atomicCAS(pv.status, 0, CF_ERR_RANGE);
        p.rows = min(max(rows, 0), line.most);
        p.left = p.length = steps_of(p.rows, kStepLog2);
    } else {
        const long long per_layer = line.length_of_layer(), total = per_layer * a.n_layers;
        size = max(a.least_share, quotient_up(total, a.n_shares));
        const long long begin = share * size, mine = min(size, total - begin);
        if (writer && !a.marks_by_unit) a.marks[share] = make_int4(0, 0, 0, 0);
        if (share == 0 && (!together || warp == 0))
            for (int b = lane; b < pv.n_requests; b += 32)
                if (pv.rows[b] < 0 || pv.rows[b] > line.most) atomicCAS(pv.status, 0, CF_ERR_RANGE);
        if (mine <= 0) return;                               // a warp's or the whole CTA's, no barrier follows
        p = line.find(begin, mine, per_layer);
    }
    const uint32_t ring = smem_u32(s_ring) + warp * kRing, bars = smem_u32(s_bars + warp * kStages);
    if (lane == 0) s_walk[warp] = p, s_next[warp] = p.first_step(cost) + first_step;
    Feeder<D> feeder = {pv, a, line, s_walk + warp, s_next + warp, first_step, stride, lane, 0, 0, nullptr, 0, ring, bars, 0u, false};
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) feeder.feed();
    unsigned taken = 0;                                      // steps that were waited for
    bool given_up = false;                                   // a wait ran out: no copies are issued any more, and none waited for
    unsigned lost = 0;                                       // which copy did not come
    const uint32_t code_lane = g * (D / 2) + t * (D / 8);    // a lane's codes within the rows of its half, keys and values alike
    const uint32_t scale_lane = g * (D / 16) + (FEW ? 4 * t % (D / 16) : 0);

    for (; p.left > 0; line.next_unit(p)) {                  // a unit, or the share's part of one
        const int start = p.first_step(cost), last = p.last_step(cost);
        if (last <= start) continue;                         // the unit's first step is the next share's
        const int head = a.tiles.quotient(p.unit), col0 = (p.unit - head * (int)a.tiles.d) * kCols;
        // the queries: lane (g, t) holds dims 32 j + 8 t .. + 7 of its column of the products, g (FEW: those of group g % kGroups of
        // query column g / kGroups, zeros elsewhere)
        uint32_t qf[NT][kParts][kGroups][2][2];
        float cs[kOwn];                                      // what turns sums of codes into base-2 logits
        int sees[kOwn];                                      // rows that the lane's queries see
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int column = col0 + (FEW ? g / kGroups : 8 * n + g);
            constexpr int kLoads = FEW ? 1 : kGroups;
            float x[kLoads][8];
            uint32_t amax = 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
            if (column < a.columns) {
                const int token = a.group.quotient(column), h = head * (int)a.group.d + a.group.remainder(column);
                const T* q = static_cast<const T*>(a.q) + (size_t)p.layer * a.q_layer_stride + (((size_t)p.request * a.q_len + token) * a.n_q_heads + h) * D +
                             8 * t + (FEW ? 32 * (g % kGroups) : 0);
#pragma unroll
                for (int j = 0; j < kLoads; ++j) {
                    uint32_t w[4 * kParts];
#pragma unroll
                    for (int i = 0; i < kParts; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = *reinterpret_cast<const uint4*>(q + 32 * j + 4 * i);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[j][i] = IsF32<T>::value ? __uint_as_float(w[i % (4 * kParts)]) : i & 1 ? bf16_high(w[i / 2]) : bf16_low(w[i / 2]);
                        amax = max(amax, __float_as_uint(x[j][i]) & 0x7fffffffu);
                    }
                }
            }
#pragma unroll
            for (int y = 1; y < (FEW ? 4 * kGroups : 4); y <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, y));
            int e = amax == 0 || amax >= 0x7f800000u ? 0 : (int)(amax >> 23) - 127;      // the largest magnitude comes to lie in [1, 2)
            e = max(-126, min(126, e));
            const float down = __int_as_float((127 - e) << 23), up = __int_as_float((127 + e) << 23);
#pragma unroll
            for (int j = 0; j < kGroups; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool mine = !FEW || j == g % kGroups;
                    const float lo = mine ? x[j % kLoads][2 * i] * down : 0.f, hi = mine ? x[j % kLoads][2 * i + 1] * down : 0.f;
                    qf[n][0][j][i / 2][i & 1] = pack_f16(lo, hi);
                    if (kParts == 2) qf[n][kParts - 1][j][i / 2][i & 1] = pack_f16_rest(lo, hi, qf[n][0][j][i / 2][i & 1]);
                }
#pragma unroll
            for (int i = 0; i < (FEW ? 1 : 2); ++i) {
                cs[FEW ? 0 : 2 * n + i] = a.scale_log2 * __shfl_sync(0xffffffffu, up, (2 * t + i) * 4);
                const int mine = col0 + (FEW ? 2 * t / kGroups : 8 * n + 2 * t + i);
                sees[FEW ? 0 : 2 * n + i] = mine < a.columns ? p.rows - a.q_len + 1 + a.group.quotient(mine) : p.rows;
            }
        }
        const int all_see = p.rows - a.q_len + 1 + a.group.quotient(col0);       // what the tile's first column sees, the fewest

        // base: what logits are taken from (the running maximum, 0 before there is one); slack: how far above it they may lie
        float o[NT][kGroups][2][4], base[kOwn], slack[kOwn], l[kOwn];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < kGroups; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[n][j][i][k] = 0.f;
#pragma unroll
        for (int c = 0; c < kOwn; ++c) base[c] = 0.f, slack[c] = -INFINITY, l[c] = 0.f;
        int exponent = kLeastExponent;                       // values are taken in units of 2^(exponent - kHead)
        uint32_t scale_limit = (uint32_t)(127 + exponent) * 0x00800080u;   // 2^exponent as bf16, twice
        float scale_down = power_of_two(kHead - exponent);

        for (int step = start + first_step; step < last; step += stride) {
            const uint32_t stage = taken % kStages, blocks = ring + stage * kStepBlocks * kBytes;
            const bool came = given_up || tc::mbar_wait(bars + 8 * stage, taken / kStages & 1, &s_abort, a.wait_limit);
            ++taken;
            // S^T of 32 keys: s[block][half][own column]
            float s[kStepBlocks][2][kOwn];
#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x) {
                const uint32_t codes = blocks + x * kBytes + code_lane, scales = blocks + x * kBytes + scale_lane;
                uint32_t k0[kGroups], k1[kGroups], ks[2][kScaleWords];
                lds<kGroups>(codes + key_code_at<D>(0), k0);
                lds<kGroups>(codes + key_code_at<D>(8), k1);
#pragma unroll
                for (int h = 0; h < 2; ++h) lds<kScaleWords>(scales + key_scale_at<D>(8 * h), ks[h]);
                float c[NT][4];
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    const uint32_t a00 = two_numbers<0>(k0[j]), a10 = two_numbers<0>(k1[j]), a20 = two_numbers<1>(k0[j]), a30 = two_numbers<1>(k1[j]);
                    const uint32_t a01 = two_numbers<2>(k0[j]), a11 = two_numbers<2>(k1[j]), a21 = two_numbers<3>(k0[j]), a31 = two_numbers<3>(k1[j]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (FEW && j > 0) mma_f16(c[n], a00, a10, a20, a30, qf[n][0][j][0][0], qf[n][0][j][0][1]);
                        else mma_f16_first(c[n], a00, a10, a20, a30, qf[n][0][j][0][0], qf[n][0][j][0][1]);
                        mma_f16(c[n], a01, a11, a21, a31, qf[n][0][j][1][0], qf[n][0][j][1][1]);
                        if (kParts == 2) {
                            mma_f16(c[n], a00, a10, a20, a30, qf[n][kParts - 1][j][0][0], qf[n][kParts - 1][j][0][1]);
                            mma_f16(c[n], a01, a11, a21, a31, qf[n][kParts - 1][j][1][0], qf[n][kParts - 1][j][1][1]);
                        }
                        if (!FEW) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float f = j & 1 ? bf16_high(ks[h][j / 2 % kScaleWords]) : bf16_low(ks[h][j / 2 % kScaleWords]);
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    float& y = s[x][h][(2 * n + i) % kOwn];
                                    y = j == 0 ? c[n][2 * h + i] * f : fmaf(c[n][2 * h + i], f, y);
                                }
                            }
                        }
                    }
                }
                if (FEW) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float y = fmaf(c[0][2 * h + 1], bf16_high(ks[h][0]), c[0][2 * h] * bf16_low(ks[h][0]));
                        if (kGroups == 4) y += __shfl_xor_sync(0xffffffffu, y, 1);
                        s[x][h][0] = y;
                    }
                }
            }
            uint32_t ws[kStepBlocks][2][kScaleWords];        // scales of the values of keys g and g + 8
#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                for (int h = 0; h < 2; ++h) lds<kScaleWords>(blocks + x * kBytes + scale_lane + value_scale_at<D>(8 * h), ws[x][h]);

#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < kOwn; ++c) s[x][h][c] = fmaf(s[x][h][c], cs[c], -base[c]);
            if ((step + 1) * kStepRows > all_see) {          // some query does not see some of the keys
                bool nan = false;
#pragma unroll
                for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = step * kStepRows + x * kBlockRows + g + 8 * h;
#pragma unroll
                        for (int c = 0; c < kOwn; ++c)
                            if (row >= sees[c]) s[x][h][c] = -INFINITY;
#pragma unroll
                        for (int i = 0; i < kScaleWords; ++i) {
                            if (row >= p.rows) ws[x][h][i] = 0u;     // rows behind the last may hold anything
                            nan |= bf16_low(ws[x][h][i]) != bf16_low(ws[x][h][i]) || bf16_high(ws[x][h][i]) != bf16_high(ws[x][h][i]);
                        }
                    }
                if (__any_sync(0xffffffffu, nan)) {          // a NaN reaches the queries that see its row, and no others
#pragma unroll
                    for (int j = 0; j < 2 * kScaleWords; ++j) {
                        bool is_nan[kStepBlocks][2];
#pragma unroll
                        for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float y = j & 1 ? bf16_high(ws[x][h][j / 2]) : bf16_low(ws[x][h][j / 2]);
                                is_nan[x][h] = y != y;
                                if (is_nan[x][h]) ws[x][h][j / 2] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
                            }
#pragma unroll
                        for (int c = 0; c < kOwn; ++c) {
                            bool hit = false;
#pragma unroll
                            for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                                for (int h = 0; h < 2; ++h) hit |= is_nan[x][h] && step * kStepRows + x * kBlockRows + g + 8 * h < sees[c];
                            // lanes of the same columns: bits t, t + 4, ...
                            if (__ballot_sync(0xffffffffu, hit) & (0x11111111u << t)) {
                                const float bad = __int_as_float(0x7fffffff);
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    if (!FEW) {
                                        o[c / 2][j % kGroups][k][c & 1] = o[c / 2][j % kGroups][k][(c & 1) + 2] = bad;
                                    } else {
#pragma unroll
                                        for (int jj = 0; jj < kGroups; ++jj) o[0][jj][k][j & 1] = o[0][jj][k][(j & 1) + 2] = bad;
                                    }
                                }
                            }
                        }
                    }
                }
            }
            bool raise = !came;                              // one vote for what is rare
#pragma unroll
            for (int c = 0; c < kOwn; ++c) raise |= fmaxf(fmaxf(s[0][0][c], s[0][1][c]), fmaxf(s[1][0][c], s[1][1][c])) > slack[c];
            uint32_t most = scale_limit;                     // scales order as integers
#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                for (int i = 0; i < kScaleWords; ++i) most = __vmaxu2(most, __vmaxu2(ws[x][0][i], ws[x][1][i]));
            raise |= most != scale_limit;
            if (__any_sync(0xffffffffu, raise)) {
                if (__any_sync(0xffffffffu, !came)) given_up = true, lost = taken - 1;
                float vmax = 0.f;
#pragma unroll
                for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < kScaleWords; ++i) vmax = fmaxf(vmax, fmaxf(bf16_low(ws[x][h][i]), bf16_high(ws[x][h][i])));
#pragma unroll
                for (int y = 1; y < 32; y <<= 1) vmax = fmaxf(vmax, __shfl_xor_sync(0xffffffffu, vmax, y));
                float f = 1.f;
                if (vmax > bf16_low(scale_limit)) {
                    const int e = min((int)(__float_as_uint(vmax) >> 23) - 126, 127);
                    f = exp2_fast((float)(exponent - e));
                    exponent = e;
                    scale_limit = (uint32_t)(127 + e) * 0x00800080u;
                    scale_down = power_of_two(kHead - e);
                }
#pragma unroll
                for (int c = 0; c < kOwn; ++c) {
                    float y = -INFINITY;                     // above `base`
#pragma unroll
                    for (int x = 0; x < kStepBlocks; ++x) y = fmaxf(y, fmaxf(s[x][0][c], s[x][1][c]));
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, k));
                    float r = 1.f;
                    if (slack[c] != -INFINITY) y = fmaxf(y, 0.f), r = exp2_fast(-y);
                    if (y != -INFINITY) {                    // otherwise the column has seen nothing yet
                        base[c] += y;
                        slack[c] = kSlack;
#pragma unroll
                        for (int x = 0; x < kStepBlocks; ++x) s[x][0][c] -= y, s[x][1][c] -= y;
                    }
                    l[c] *= r;
#pragma unroll
                    for (int j = 0; j < kGroups; ++j)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            o[c / 2][j][k][c & 1] *= r * f, o[c / 2][j][k][(c & 1) + 2] *= r * f;
                            if (FEW) o[0][j][k][1] *= r * f, o[0][j][k][3] *= r * f;
                        }
                }
            }
            // the probabilities
#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < kOwn; ++c) {
                        const float y = exp2_fast(s[x][h][c]);
                        l[c] += y;
                        s[x][h][c] = y * scale_down;
                    }
            // O^T += V^T P^T, group by group
#pragma unroll
            for (int x = 0; x < kStepBlocks; ++x) {
                uint32_t vw[2][kGroups];                     // [half]: groups two by two of an even key's codes, of an odd one's
                uint32_t b[NT][kParts][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) lds<kGroups>(blocks + x * kBytes + code_lane + value_code_at<D>(8 * h, 0), vw[h]);
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    constexpr uint32_t kLow = 0x0f0f0f0fu;
                    uint32_t even[2], odd[2];                // [half]: codes of an even dim of two keys to a byte; of an odd dim
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w0 = vw[h][j / 2], w1 = vw[h][kGroups / 2 + j / 2];
                        even[h] = (w0 & kLow) | ((w1 << 4) & ~kLow);
                        odd[h] = ((w0 >> 4) & kLow) | (w1 & ~kLow);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (!FEW || j == 0) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t w = ws[x][h][FEW ? 0 : j / 2 % kScaleWords];
                                const float v0 = FEW || !(j & 1) ? bf16_low(w) : bf16_high(w), v1 = FEW ? bf16_high(w) : v0;
                                const float p0 = s[x][h][2 * n % kOwn] * v0, p1 = s[x][h][(2 * n + 1) % kOwn] * v1;
                                const uint32_t packed = pack_f16(p0, p1);
                                b[n][0][h] = transposed(packed);
                                if (kParts == 2) b[n][kParts - 1][h] = transposed(pack_f16_rest(p0, p1, packed));
                            }
                        }
#pragma unroll
                        for (int i = 0; i < kParts; ++i) {
                            if (j & 1) {
                                mma_f16(o[n][j][0], two_numbers<2>(even[0]), two_numbers<2>(odd[0]), two_numbers<2>(even[1]), two_numbers<2>(odd[1]), b[n][i][0], b[n][i][1]);
                                mma_f16(o[n][j][1], two_numbers<3>(even[0]), two_numbers<3>(odd[0]), two_numbers<3>(even[1]), two_numbers<3>(odd[1]), b[n][i][0], b[n][i][1]);
                            } else {
                                mma_f16(o[n][j][0], two_numbers<0>(even[0]), two_numbers<0>(odd[0]), two_numbers<0>(even[1]), two_numbers<0>(odd[1]), b[n][i][0], b[n][i][1]);
                                mma_f16(o[n][j][1], two_numbers<1>(even[0]), two_numbers<1>(odd[0]), two_numbers<1>(even[1]), two_numbers<1>(odd[1]), b[n][i][0], b[n][i][1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();                                    // the stage has been read
            if (!given_up) feeder.feed();
        }

        // the unit is done, or as much of it as the share has
        const float unit_scale = power_of_two(exponent - kHead);
        float m[kOwn];
#pragma unroll
        for (int c = 0; c < kOwn; ++c) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[c] += __shfl_xor_sync(0xffffffffu, l[c], x);
            m[c] = slack[c] == -INFINITY ? -INFINITY : base[c];
        }
        const bool begins = p.at <= cost, whole = begins && p.end() == p.length;
        const int slot = 2 * share + (begins ? 1 : 0);
        // a lane's dims 32 j + 4 g .. + 3 of own column c, where it has them
        auto has = [&](int j) { return !FEW || t % (kGroups / 2) == j / 2; };
        auto dims = [&](int c, int j, float f) {
            const int n = FEW ? 0 : c / 2, i = FEW ? j & 1 : c & 1;
            return make_float4(o[n][j][0][i] * f, o[n][j][0][i + 2] * f, o[n][j][1][i] * f, o[n][j][1][i + 2] * f);
        };
        auto tile_column = [&](int c) { return FEW ? 2 * t / kGroups : 8 * (c / 2) + 2 * t + (c & 1); };
        const bool first_lane = g == 0 && (!FEW || t % (kGroups / 2) == 0);      // of those that have a column
        if (together) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int c = tile_column(i);
                float* row = s_o + (warp * kCols + c) * kOStride + 4 * g;
#pragma unroll
                for (int j = 0; j < kGroups; ++j)
                    if (has(j)) *reinterpret_cast<float4*>(row + 32 * j) = dims(i, j, unit_scale);
                if (first_lane) s_m[warp * kCols + c] = m[i], s_l[warp * kCols + c] = l[i];
            }
            __syncthreads();
            for (int i = tid; i < kCols * (D / 4); i += kThreads) {
                const int c = i / (D / 4), d = i % (D / 4) * 4, column = col0 + c;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w * kCols + c]);
                float sum = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float mw = s_m[w * kCols + c], lw = s_l[w * kCols + c];
                    const float4 y = *reinterpret_cast<const float4*>(s_o + (w * kCols + c) * kOStride + d);
                    const float k = mw == top ? 1.f : exp2_fast(mw - top);       // a warp that saw no key has zeros
                    sum = fmaf(lw, k, sum);
                    x.x = fmaf(y.x, k, x.x), x.y = fmaf(y.y, k, x.y), x.z = fmaf(y.z, k, x.z), x.w = fmaf(y.w, k, x.w);
                }
                if (n_cluster > 1) {                         // for the cluster, where the ring was
                    *reinterpret_cast<float4*>(s_part + c * D + d) = x;
                    if (d == 0) s_part_ml[c] = top, s_part_ml[kCols + c] = sum;
                } else if (whole) {
                    if (column < a.columns) {
                        const float inv = sum == 0.f ? 0.f : reciprocal(sum);
                        store4<T>(out_row<T, D>(a, p.layer, p.request, head, column) + d, x.x * inv, x.y * inv, x.z * inv, x.w * inv);
                        if (d == 0) store_lse(a, pv.n_requests, p.layer, p.request, head, column, top, sum);
                    }
                } else {
                    *reinterpret_cast<float4*>(a.part_o + ((size_t)slot * kCols + c) * D + d) = x;
                    if (d == 0) a.part_ml[(size_t)slot * 2 * kCols + c] = top, a.part_ml[(size_t)slot * 2 * kCols + kCols + c] = sum;
                }
            }
            if (n_cluster > 1) {                             // the CTAs join their results, each a part of the dims
                tc::cluster_sync();
                for (int i = rank * kThreads + tid; i < kCols * (D / 4); i += n_cluster * kThreads) {
                    const int c = i / (D / 4), d = i % (D / 4) * 4, column = col0 + c;
                    Part x = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
                    for (int k = 0; k < n_cluster; ++k)
                        x.add(cluster_load(s_part_ml + c, k), cluster_load(s_part_ml + kCols + c, k), cluster_load4(s_part + c * D + d, k));
                    if (column < a.columns) {
                        const float inv = x.sum == 0.f ? 0.f : reciprocal(x.sum);
                        store4<T>(out_row<T, D>(a, p.layer, p.request, head, column) + d, x.x.x * inv, x.x.y * inv, x.x.z * inv, x.x.w * inv);
                        if (d == 0) store_lse(a, pv.n_requests, p.layer, p.request, head, column, x.top, x.sum);
                    }
                }
                tc::cluster_sync();                          // everyone has read
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int c = tile_column(i), column = col0 + c;
                if (whole) {
                    if (column < a.columns) {
                        const float f = l[i] == 0.f ? 0.f : unit_scale * reciprocal(l[i]);
                        T* row = out_row<T, D>(a, p.layer, p.request, head, column) + 4 * g;
#pragma unroll
                        for (int j = 0; j < kGroups; ++j)
                            if (has(j)) {
                                const float4 y = dims(i, j, f);
                                store4<T>(row + 32 * j, y.x, y.y, y.z, y.w);
                            }
                        if (first_lane) store_lse(a, pv.n_requests, p.layer, p.request, head, column, m[i], l[i]);
                    }
                } else {
                    float* row = a.part_o + ((size_t)slot * kCols + c) * D + 4 * g;
#pragma unroll
                    for (int j = 0; j < kGroups; ++j)
                        if (has(j)) *reinterpret_cast<float4*>(row + 32 * j) = dims(i, j, unit_scale);
                    if (first_lane) a.part_ml[(size_t)slot * 2 * kCols + c] = m[i], a.part_ml[(size_t)slot * 2 * kCols + kCols + c] = l[i];
                }
            }
        }
        if (n_cluster == 0 && writer && begins && (!whole || a.marks_by_unit)) {
            const long long more = p.length - p.end();        // of the unit in later shares
            const int lb = p.layer * pv.n_requests + p.request;
            a.marks[a.marks_by_unit ? lb * line.units + p.unit : share] = make_int4(whole ? 0 : 1 + (int)quotient_up(more, size), share, lb, p.unit);
        }
    }
    if (given_up) {                                          // its copies in flight are given the time to end
        for (; lost < feeder.issued; ++lost) {
            const long long t0 = clock64();
            while (!tc::mbar_try_wait(bars + 8 * (lost % kStages), lost / kStages & 1) && clock64() - t0 < tc::kWaitLimitCycles) {}
        }
        if (lane == 0) atomicCAS(pv.status, 0, CF_ERR_TIMEOUT);
    }
}

constexpr int kAtOnce = 4;                        // parts whose loads are under way together

// Joins the parts of the units that were cut: a block per mark and `cols` of the unit's columns, whose threads have a column's
// four dims each and, where that leaves some, every n-th part.  Joining a unit of a hundred parts in one block took 12 us (a
// request of 24 000 rows, 28/4 heads: 31 us a call).
template <typename T, int D>
__global__ void __launch_bounds__(kMergeThreads)
kv4_merge_kernel(Kv4Args args, PagesView pv, Divisor requests, int tile, int cols, int lanes_log2) {
    chain_next();
    __shared__ Part s_part[kMergeThreads];
    chain_wait();
    const Kv4Args& a = args;
    const int4 mark = a.marks[blockIdx.x];
    if (mark.x > 0) {
        const int lanes = 1 << lanes_log2, n = kMergeThreads >> lanes_log2;       // a column's dims have D/4 lanes
        const int k0 = threadIdx.x >> lanes_log2, i = threadIdx.x & (lanes - 1), c = blockIdx.y * cols + i / (D / 4), d = i % (D / 4) * 4;
        const int head = a.tiles.quotient(mark.w), column = (mark.w - head * (int)a.tiles.d) * tile + c;
        Part x = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int k = k0; k < mark.x; k += n * kAtOnce) {
            float m[kAtOnce], l[kAtOnce];
            float4 y[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int part = min(k + j * n, mark.x - 1);
                const size_t slot = part == 0 ? 2 * (size_t)mark.y + 1 : 2 * (size_t)(mark.y + part);
                m[j] = a.part_ml[slot * 2 * tile + c], l[j] = a.part_ml[slot * 2 * tile + tile + c];
                y[j] = *reinterpret_cast<const float4*>(a.part_o + (slot * tile + c) * D + d);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (k + j * n < mark.x) x.add(m[j], l[j], y[j]);
        }
        if (n > 1) {
            s_part[threadIdx.x] = x;
            __syncthreads();
        }
        if (k0 == 0 && column < a.columns) {
            for (int k = 1; k < n; ++k) {
                const Part& y = s_part[k * lanes + i];
                x.add(y.top, y.sum, y.x);
            }
            const int layer = requests.quotient(mark.z), request = mark.z - layer * pv.n_requests;
            const float inv = x.sum == 0.f ? 0.f : reciprocal(x.sum);
            store4<T>(out_row<T, D>(a, layer, request, head, column) + d, x.x.x * inv, x.x.y * inv, x.x.z * inv, x.x.w * inv);
            if (d == 0) store_lse(a, pv.n_requests, layer, request, head, column, x.top, x.sum);
        }
    }
}

// How a call is cut: everything the host can know of it.
struct Cut {
    bool tc;                                      // the tensor-core kernel
    int nt;                                       // products of eight columns that a warp takes
    bool few;
    int tile, tiles, columns;                     // columns of a unit, units and columns of a kv head
    int warps, ctas, n_shares, warps_per_share;
    int cluster;                                  // CTAs of a unit, 0: shares of the line
    int marks;                                    // units, or shares where they are fewer
    bool marks_by_unit;
};

Cut cut_of(const cf_geom* g, const cf_pages* p, int q_len, int n_layers) {
    Cut c = {};
    c.columns = g->n_q_heads / g->n_kv_heads * q_len;
    c.nt = c.columns <= 8 ? 1 : 2;
    c.few = c.columns <= tile_columns(g->head_dim, 1, true);
    c.tile = tile_columns(g->head_dim, c.nt, c.few);
    const double heads = (double)n_layers * p->n_requests * g->n_kv_heads;
    c.tc = kv4_attn_tc_supported(g, c.columns, heads * ((c.columns + kTcColumns - 1) / kTcColumns));
    if (c.tc) c.tile = kTcColumns;
    c.tiles = (c.columns + c.tile - 1) / c.tile;
    c.warps = warps_of(c.few);
    c.ctas = sm_count() * ctas_per_sm(c.nt, c.few);
    // A CTA's warps pay for every unit of a share of theirs with a barrier and a join, about 16 steps of the line; warps with shares
    // of their own with 3 steps for every unit and every share.  With U units and W warps: 16 U against 3 (U + W).
    // Measured (together / alone, us): 96 requests, 28/4 (U = 0.22 W) 46.7 / 44.9; 512 short ones, 32/8 (2.3 W) 94.6 / 39.4;
    // 3 requests, four layers, 32/8 (0.05 W) 17.3 / 21.2; 8 long ones, 32/32 (0.11 W) 122 / 126.
    const double units = heads * c.tiles;
    c.warps_per_share = 5.0 * units >= (double)c.ctas * c.warps ? 1 : c.warps;
    c.n_shares = c.warps_per_share == 1 ? c.ctas * c.warps : c.ctas;
    if (c.tc) {                                   // a share to a CTA, one to an SM
        c.ctas = c.n_shares = sm_count();
        c.warps_per_share = c.warps;
    }
    else {
        // Short caches, by the room that the table has: units that fit the device at once, with few steps for a warp, have a cluster
        // each, which joins its results without a second launch.  Measured (shares of the line / clusters, us, lengths of half to all of
        // the room): 12/2 heads, one request of 500, 1000, 2000, 4000, 8000 rows 8.2 / 6.2, 8.5 / 6.2, 8.7 / 7.1, 8.7 / 8.5, 9.0 / 11.5
        // (eight steps a warp); 28/4, eight requests of up to that 10.1 / 7.8, 10.7 / 8.0, 11.6 / 9.2, 12.1 / 11.6, 15.1 / 16.2 (eight);
        // a column a head, 32/32, one of 2000, 4000, 8000 10.6 / 7.9, 11.8 / 9.8, 15.0 / 12.9, two of 4000, 8000 13.3 / 12.0, 19.3 / 19.7
        // (eight steps), four of 4000 20.1 / 19.7 (eight), eight of 1000, 2000, 4000 15.3 / 11.0, 21.4 / 18.9 (nine), 30.0 / 30.4 (sixteen);
        // with the whole of six steps, 12/2, one of 6144 8.3 / 9.7, 28/4, eight of them 13.3 / 13.8, of nine with few columns, 2/2, one of
        // 18432 10.4 / 13.8.  It is the room that counts, not the rows: with room for 32768, 12/2, one of 1011 8.3 instead of 5.9,
        // 28/4, eight of 1000 10.5 instead of 7.7, 32/32, one of 2000 10.6 instead of 7.8.
        const double steps = ((double)p->table_cols * p->page_rows + kStepRows - 1) / kStepRows;
        int cluster = 1;
        while (cluster < kMostCluster && cluster * c.warps < steps && 2 * units * cluster <= c.ctas) cluster *= 2;
        if (units * cluster <= c.ctas && steps <= (c.few ? kClusterStepsFew : kClusterSteps) * cluster * c.warps) {
            c.cluster = cluster;
            c.warps_per_share = c.warps;
            c.ctas = (int)units * cluster;
        }
    }
    c.marks_by_unit = units <= c.n_shares;
    c.marks = c.marks_by_unit ? (int)units : c.n_shares;
    return c;
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

int check_attn(const cf_geom* geom, const cf_pages* pages, int q_len, int n_layers) {
    int rc = validate(geom, nullptr);
    if (rc == CF_OK) rc = check_pages(pages);
    if (rc != CF_OK) return rc;
    if (q_len <= 0 || n_layers <= 0 || n_layers > 65535) return CF_ERR_INVALID_ARG;
    const long long columns = (long long)geom->n_q_heads / geom->n_kv_heads * q_len;
    if ((long long)n_layers * pages->n_requests > INT_MAX) return CF_ERR_INVALID_ARG;
    const long long tiles = columns / 2 + 1;      // at least as many as cut_of makes
    if (columns > (1 << 24) || tiles * geom->n_kv_heads * ((long long)pages->table_cols * (pages->page_rows / 16) / kStepBlocks + 2 + kMostCost) > INT_MAX)
        return CF_ERR_INVALID_ARG;                // a request's part of the line is counted in 32 bits
    return CF_OK;
}

size_t attn_smem(int head_dim, int warps, int tile) {
    return (size_t)warps * kStages * kStepBlocks * block_bytes(head_dim) + (size_t)warps * tile * (head_dim + 4) * 4 + 2 * (size_t)warps * tile * 4 +
           (size_t)warps * kStages * 8;
}

template <typename T, int D>
int launch_merge(const Kv4Args& a, const PagesView& pv, int tile, int marks, cudaStream_t stream) {
    // a block takes all columns of a unit where units are many, fewer where they are not
    int cols = std::min(tile, kMergeThreads / (D / 4));
    while (cols > 1 && marks * (tile / cols) < 2 * sm_count()) cols /= 2;
    int lanes_log2 = 0;
    while (1 << lanes_log2 < cols * (D / 4)) ++lanes_log2;
    return launch_chained(kv4_merge_kernel<T, D>, dim3((unsigned)marks, (unsigned)(tile / cols)), kMergeThreads, 0, stream, a, pv,
                          Divisor(pv.n_requests), tile, cols, lanes_log2);
}

template <typename T, int D, int NT, bool FEW>
int launch_attn(const Kv4Args& a, const PagesView& pv, const Cut& c, cudaStream_t stream) {
    static PerDeviceOnce once;
    const size_t smem = attn_smem(D, warps_of(FEW), tile_columns(D, NT, FEW));
    const int rc = configure_smem_once(once, kv4_attn_kernel<T, D, NT, FEW>, (int)smem);
    if (rc != CF_OK) return rc;
    const int err = launch_chained_clusters(kv4_attn_kernel<T, D, NT, FEW>, dim3((unsigned)c.ctas), 32 * warps_of(FEW), smem, (unsigned)std::max(1, c.cluster),
                                            stream, a, pv);
    return err != CF_OK || c.cluster > 0 ? err : launch_merge<T, D>(a, pv, c.tile, c.marks, stream);
}

template <typename T, int D>
int launch_attn_cut(const Kv4Args& a, const PagesView& pv, const Cut& c, cudaStream_t stream) {
    if (c.few) return launch_attn<T, D, 1, true>(a, pv, c, stream);
    return c.nt == 1 ? launch_attn<T, D, 1, false>(a, pv, c, stream) : launch_attn<T, D, 2, false>(a, pv, c, stream);
}

template <typename T>
int launch_attn_typed(const Kv4Args& a, const PagesView& pv, const Cut& c, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_attn_cut<T, 128>(a, pv, c, stream) : launch_attn_cut<T, 64>(a, pv, c, stream);
}

int run_attn(const cf_geom* geom, const cf_pages* pages, int32_t n_layers, int32_t q_len, const void* q, int64_t q_layer_stride, const void* kv4,
             int64_t kv4_layer_stride, float softmax_scale, void* out, int64_t out_layer_stride, float* lse, void* workspace, size_t workspace_bytes,
             int wait_limit, bool copies, void* stream) {
    const int rc = check_attn(geom, pages, q_len, n_layers);
    if (rc != CF_OK) return rc;
    if (!q || !kv4 || !out || !workspace) return CF_ERR_INVALID_ARG;
    const int esize = geom->dtype == CF_BF16 ? 2 : 4;
    for (const void* p : {q, kv4, static_cast<const void*>(out)})
        if (reinterpret_cast<uintptr_t>(p) % 16) return CF_ERR_INVALID_ARG;
    if ((q_layer_stride * esize) % 16 || (out_layer_stride * esize) % 16 || kv4_layer_stride % 16) return CF_ERR_INVALID_ARG;
    const long long layer_elems = (long long)pages->n_requests * q_len * geom->n_q_heads * geom->head_dim;
    if (n_layers > 1 && (q_layer_stride < layer_elems || out_layer_stride < layer_elems ||
                         kv4_layer_stride < (long long)cf_kv4_layer_bytes(geom, pages)))
        return CF_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < cf_kv4_attn_workspace_bytes(geom, pages, q_len, n_layers))
        return CF_ERR_WORKSPACE;
    const Cut c = cut_of(geom, pages, q_len, n_layers);
    const float scale = softmax_scale != 0.f ? softmax_scale : 1.f / sqrtf((float)geom->head_dim);
    const size_t rows = 2 * (size_t)c.n_shares * c.tile;
    char* w = static_cast<char*>(workspace);
    Kv4Args a = {};
    a.q = q, a.kv4 = static_cast<const unsigned char*>(kv4), a.out = out, a.lse = lse;
    a.part_o = reinterpret_cast<float*>(w);
    a.part_ml = reinterpret_cast<float*>(w + round_up(rows * geom->head_dim * 4));
    a.marks = reinterpret_cast<int4*>(w + round_up(rows * geom->head_dim * 4) + round_up(rows * 8));
    a.q_layer_stride = q_layer_stride, a.kv4_layer_stride = kv4_layer_stride, a.out_layer_stride = out_layer_stride;
    a.n_layers = n_layers, a.q_len = q_len, a.n_q_heads = geom->n_q_heads, a.n_kv_heads = geom->n_kv_heads;
    a.columns = c.columns;
    a.group = Divisor(geom->n_q_heads / geom->n_kv_heads), a.tiles = Divisor(c.tiles), a.blocks_per_page = Divisor(pages->page_rows / kBlockRows);
    a.n_shares = c.n_shares, a.warps_per_share = c.warps_per_share, a.marks_by_unit = c.marks_by_unit;
    a.least_share = c.warps_per_share == 1 ? kLeastAlone : kLeastTogether;
    a.unit_cost = c.warps_per_share == 1 ? kCostAlone : kCostTogether;
    if (c.tc) a.least_share = kLeastTc, a.unit_cost = kCostTc;
    if (c.cluster > 0) {
        a.unit_cost = 0;
        a.cluster = Divisor(c.cluster), a.units_of = Divisor(geom->n_kv_heads * c.tiles), a.requests = Divisor(pages->n_requests);
    }
    a.scale_log2 = scale * kLog2e;
    a.no_copies = !copies, a.wait_limit = wait_limit;
    const PagesView pv = make_pages_view(pages);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (c.tc) {
        const int err = launch_kv4_attn_tc(a, pv, s);
        return err != CF_OK ? err : launch_merge<__nv_bfloat16, 128>(a, pv, c.tile, c.marks, s);
    }
    return geom->dtype == CF_BF16 ? launch_attn_typed<__nv_bfloat16>(a, pv, c, geom->head_dim, s)
                                  : launch_attn_typed<float>(a, pv, c, geom->head_dim, s);
}

}  // namespace

}  // namespace cf

using namespace cf;

extern "C" {

size_t cf_kv4_attn_workspace_bytes(const cf_geom* geom, const cf_pages* pages, int32_t q_len, int32_t n_layers) {
    if (check_attn(geom, pages, q_len, n_layers) != CF_OK) return 0;
    const Cut c = cut_of(geom, pages, q_len, n_layers);
    const size_t rows = 2 * (size_t)c.n_shares * c.tile;
    return round_up(rows * geom->head_dim * 4) + round_up(rows * 8) + round_up((size_t)c.marks * sizeof(int4));
}

int cf_kv4_attn(const cf_geom* geom, const cf_pages* pages, int32_t n_layers, int32_t q_len, const void* q,
                int64_t q_layer_stride, const void* kv4, int64_t kv4_layer_stride, float softmax_scale, void* out,
                int64_t out_layer_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return run_attn(geom, pages, n_layers, q_len, q, q_layer_stride, kv4, kv4_layer_stride, softmax_scale, out, out_layer_stride, lse, workspace,
                    workspace_bytes, (int)tc::kWaitLimitCycles, true, stream);
}

int cf_debug_kv4_attn(const cf_geom* geom, const cf_pages* pages, int32_t n_layers, int32_t q_len, const void* q,
                      int64_t q_layer_stride, const void* kv4, int64_t kv4_layer_stride, float softmax_scale, void* out,
                      int64_t out_layer_stride, float* lse, void* workspace, size_t workspace_bytes, int64_t limit_cycles,
                      int32_t copies, void* stream) {
    if (limit_cycles <= 0 || limit_cycles > tc::kWaitLimitCycles) return CF_ERR_INVALID_ARG;
    return run_attn(geom, pages, n_layers, q_len, q, q_layer_stride, kv4, kv4_layer_stride, softmax_scale, out, out_layer_stride, lse, workspace,
                    workspace_bytes, (int)limit_cycles, copies != 0, stream);
}

int cf_debug_kv4_attn_kernel(const cf_geom* geom, const cf_pages* pages, int32_t q_len, int32_t n_layers, int32_t* which) {
    const int rc = check_attn(geom, pages, q_len, n_layers);
    if (rc != CF_OK) return rc;
    if (!which) return CF_ERR_INVALID_ARG;
    const Cut c = cut_of(geom, pages, q_len, n_layers);
    *which = c.tc ? 3 : c.cluster > 0 ? 2 : c.warps_per_share == 1 ? 0 : 1;
    return CF_OK;
}

}  // extern "C"
