// Attention of drafted trees over a paged cache.
//
// With s_p = scale q.k_p over the places p that a token sees, out = sum_p e^{s_p - m} v_p / sum_p e^{s_p - m} for any m; m is a
// running reference near the maximum of the scores so far, and sums made under an older one are scaled by e^{m_old - m}: one pass over
// the keys and values, each read once for up to 128 query rows.
//
// Layout.  The rows that share a key head (a sequence's new tokens times the query heads of the group) are tiled by 16 NQ WR.  A block is
// four wavefronts: WR of them side by side on rows, WT = 4 / WR on stretches of 32 places.  A wavefront goes straight from the cache to
// the matrix cores, without shared memory:
//     S^T [16 places, 16 rows] = K Q^T        A operand: a lane's 16 bytes of a key row; B: the query row's, kept in registers
//     O^T [channels, 16 rows] += V^T P^T      B operand: the lane's own weights, as S^T's accumulators hold them; A: V turned in registers
// S^T leaves lane (r = lane % 16, g = lane / 16) the places 4 g + i of row r, and the contraction of the second product takes them in
// that order (its index is (g, tile, i)), so P needs no exchange between lanes.  A lane loads V rows 4 g + i in pieces of DP / 16 channels
// and turns eight rows by byte permutes: its MFMA number j has row index r for channel (DP / 16) r + j, so the accumulators of a lane are DP / 4
// adjacent channels of row r.
#include "cache.hpp"
#include "device_utils.hpp"
#include <algorithm>

namespace slimspec {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kStep = 32;                        // places per wavefront and step
constexpr float kLowest = -3.0e38f;              // reference of a row without scores: finite, so that differences to it are numbers
constexpr float kSlack = 8.f;                    // scores may pass the reference by this (in bits) before sums are scaled

template <bool F16>
__device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// two values rounded to the type (to nearest), the first one in the low half
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (F16) return __builtin_bit_cast(uint32_t, (f16x2){(_Float16)a, (_Float16)b});
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
template <bool F16> __device__ __forceinline__ bool not_a_number_or_infinite(uint32_t half)
{
    constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;
    return (half & kExp) == kExp;
}
template <bool F16> __device__ __forceinline__ float value_of(uint16_t b)
{
    if constexpr (F16) return (float)__builtin_bit_cast(_Float16, b);
    else return bf16_to_float(b);
}

// (largest over, sum over) the four lanes that hold a row: 16 and 32 away
__device__ __forceinline__ float row_max(float v)
{
    uint32_t a, b;
    swap_pair<16>(__float_as_uint(v), a, b);
    v = fmaxf(__uint_as_float(a), __uint_as_float(b));
    swap_pair<32>(__float_as_uint(v), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float row_sum(float v)
{
    uint32_t a, b;
    swap_pair<16>(__float_as_uint(v), a, b);
    v = __uint_as_float(a) + __uint_as_float(b);
    swap_pair<32>(__float_as_uint(v), a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// ---- the division of the work
//
// Units: one step of a block (32 WT places) for one row tile of one key head.  All units of a call, ordered by sequence, head, row tile
// and place, are cut into equal runs, one per block, whatever the sequences' lengths; a run may begin and end inside a row tile, whose pieces
// tree_merge_kernel joins.  The cut depends on the books alone, so results do not change from run to run.
struct Division { int64_t units; int blocks; };
__device__ __forceinline__ int64_t run_start(const Division &d, int block) { return d.units * block / d.blocks; }
__device__ __forceinline__ int block_of(const Division &d, int64_t unit) { return (int)(((unit + 1) * d.blocks - 1) / d.units); }

struct Tiling { int rows, places; };             // of a unit
__device__ __forceinline__ int row_tiles(const Sequence &q, int group, const Tiling &t) { return (q.tokens * group + t.rows - 1) / t.rows; }
__device__ __forceinline__ int steps_of(const Sequence &q, const Tiling &t) { return (int)(((int64_t)q.len + q.tokens + t.places - 1) / t.places); }
__device__ __forceinline__ int64_t units_of(const CacheView &c, const Sequence &q, int group, const Tiling &t)
{
    return q.tokens ? (int64_t)row_tiles(q, group, t) * steps_of(q, t) * c.heads : 0;
}

// Workspace: the division and the first unit of every sequence, for the merge; the pieces
struct TreePlan { int64_t units; int32_t blocks, pad; int64_t start[1]; };
__host__ __device__ constexpr size_t plan_bytes(int n) { return ((size_t)16 + 8 * ((size_t)n + 1) + 255) & ~(size_t)255; }
// a piece of a row tile: rows x DP sums, then the references and the weights' sums of the rows
__host__ __device__ constexpr size_t piece_floats(int rows, int dp) { return (size_t)rows * dp + 2 * (size_t)rows; }

struct Where { int64_t units; int seq; int64_t start; };
// What block `block` of at most `blocks` begins with: every thread counts the units of a stretch of sequences.  tell: block 0 writes the plan.
__device__ Where divide(const CacheView &c, const BatchView &b, int group, const Tiling &tile, Division &d, int max_blocks, int block, TreePlan *plan)
{
    __shared__ int64_t wave_sum[kWaves];
    __shared__ int64_t found_start;
    __shared__ int found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int each = (b.n + kThreads - 1) / kThreads, i0 = min(b.n, (int)threadIdx.x * each), i1 = min(b.n, i0 + each);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += units_of(c, sequence_of(c, b, i), group, tile);
    int64_t inc = mine;
    if (b.n > 1) {
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int64_t o = __shfl_up(inc, s);
            if (lane >= s) inc += o;
        }
    }
    if (threadIdx.x == 0) found = -1;
    if (b.n == 1 ? threadIdx.x == 0 : lane == 63) wave_sum[wave] = inc;
    __syncthreads();
    int64_t total = 0, before = inc - mine;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int64_t x = b.n == 1 && w ? 0 : wave_sum[w];
        if (w < wave) before += x;
        total += x;
    }
    d.units = total;
    d.blocks = (int)(total < max_blocks ? (total > 0 ? total : 1) : max_blocks);
    if (block == 0) {
        if (threadIdx.x == 0) { plan->units = total; plan->blocks = d.blocks; }
        int64_t at = before;
        for (int i = i0; i < i1; ++i) {
            plan->start[i] = at;
            at += units_of(c, sequence_of(c, b, i), group, tile);
        }
    }
    if (block < d.blocks && total > 0) {
        const int64_t u = run_start(d, block);
        if (mine > 0 && before <= u && u < before + mine) {
            int64_t at = before;
            for (int i = i0; i < i1; ++i) {
                const int64_t m = units_of(c, sequence_of(c, b, i), group, tile);
                if (u < at + m) { found = i; found_start = at; break; }
                at += m;
            }
        }
    }
    __syncthreads();
    Where w;
    w.units = total;
    w.seq = __builtin_amdgcn_readfirstlane(found);
    w.start = found_start;
    return w;
}

template <int NQ, int WR> struct TileOf { static constexpr int kRows = 16 * NQ * WR, kWT = kWaves / WR, kPlaces = kStep * kWT; };

// DP: head_dim rounded up to 64, 128 or 256; EXACT: head_dim is DP
template <bool F16, int DP, bool EXACT, int NQ, int WR>
__global__ __launch_bounds__(kThreads, DP == 256 || NQ > 1 ? 2 : 3) void tree_rows_kernel(
    CacheView c, int layer, TreeCall call, BatchView b, TreePlan *__restrict__ plan, float *__restrict__ pieces)
{
    using Tile = TileOf<NQ, WR>;
    constexpr int kWT = Tile::kWT, kKC = DP / 32, kHalves = DP == 256 ? 2 : 1, kVW = DP == 64 ? 4 : 8;   // kVW: channels of V per lane and load
    constexpr int kO = kHalves * kVW;                                                                    // accumulators (of 4) per row tile
    __shared__ __align__(16) float joint[kWT > 1 ? (kWT / 2) * WR * (kO * NQ * 256 + 2 * NQ * 64) : 4];
    const Tiling tile{Tile::kRows, Tile::kPlaces};
    const int group = call.q_heads / c.heads;
    Division div;
    Where at = divide(c, b, group, tile, div, gridDim.x, blockIdx.x, plan);
    if ((int)blockIdx.x >= div.blocks || at.units == 0) return;
    const int64_t u1 = run_start(div, blockIdx.x + 1);
    int64_t u = run_start(div, blockIdx.x);
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wt = wave / WR;
    const int D = EXACT ? DP : c.head_dim;
    const int in_page = (1 << c.page_shift) - 1;
    const float unit = fmaxf(fabsf(call.scale) * kLog2e, 1.2e-38f);    // (not 0: an unseen place's score of -infinity stays one)
    const uint32_t flip = call.scale < 0.f ? 0x80008000u : 0u;

    // byte offsets of a lane's loads from the first of 16 places.  Channels past head_dim: the row's first piece again (for K, against
    // zeros of Q; what V gives there is not stored)
    uint32_t koff[EXACT ? 1 : kKC], voff[4 * (EXACT ? 1 : kHalves)];
    const uint32_t row_bytes = 2 * (uint32_t)c.place_stride;
#pragma unroll
    for (int k = 0; k < (EXACT ? 1 : kKC); ++k) koff[k] = r * row_bytes + (32 * k + 8 * g < D ? 2 * (32 * k + 8 * g) : 0);
#pragma unroll
    for (int h = 0; h < (EXACT ? 1 : kHalves); ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) voff[4 * h + i] = (4 * g + i) * row_bytes + (128 * h + kVW * r < D ? 2 * (128 * h + kVW * r) : 0);

    bool first_piece = true;
    int seq = at.seq;
    int64_t seq_start = at.start;
    while (u < u1) {
        Sequence s = sequence_of(c, b, seq);
        int64_t seq_units = units_of(c, s, group, tile);
        while (u >= seq_start + seq_units) {
            seq_start += seq_units;
            s = sequence_of(c, b, ++seq);
            seq_units = units_of(c, s, group, tile);
        }
        const int steps = __builtin_amdgcn_readfirstlane(steps_of(s, tile)), tiles = __builtin_amdgcn_readfirstlane(row_tiles(s, group, tile));
        const int slot = __builtin_amdgcn_readfirstlane(s.slot), len = __builtin_amdgcn_readfirstlane(s.len);
        const int tokens = __builtin_amdgcn_readfirstlane(s.tokens), first = __builtin_amdgcn_readfirstlane(s.first);
        const int64_t rel = u - seq_start;
        const int per_head = __builtin_amdgcn_readfirstlane((int)(rel / steps));                          // head * tiles + row tile
        const int head = per_head / tiles, rt = per_head - head * tiles;
        const int step0 = __builtin_amdgcn_readfirstlane((int)(rel - (int64_t)per_head * steps));
        const int step1 = (int)min((int64_t)steps, step0 + (u1 - u));
        const bool whole = step0 == 0 && step1 == steps;
        const int end = len + tokens;

        // this lane's query rows
        uint4 qf[NQ][kKC];
        int row_t[NQ], row_h[NQ];
        bool row_ok[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            const int row = rt * Tile::kRows + (wr * NQ + x) * 16 + r;
            row_t[x] = row / group;
            row_h[x] = head * group + row - row_t[x] * group;
            row_ok[x] = row_t[x] < tokens;
            const uint16_t *qr = call.q + (int64_t)(first + (row_ok[x] ? row_t[x] : 0)) * call.q_token_stride + (int64_t)(row_ok[x] ? row_h[x] : 0) * call.q_head_stride;
#pragma unroll
            for (int k = 0; k < kKC; ++k) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (row_ok[x] && (EXACT || 32 * k + 8 * g < D)) v = *reinterpret_cast<const uint4 *>(qr + 32 * k + 8 * g);
                qf[x][k] = make_uint4(v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip);
            }
        }

        const int64_t head_at = (int64_t)layer * c.layer_stride + head * c.head_stride;
        const auto *entries = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(c.table + (int64_t)slot * c.slot_pages);
        // the two stretches of 16 places of a step: their page numbers (-1: none, or past the end)
        auto pages_of_step = [&](int step, int (&page)[2]) {
            const int p0 = (step * kWT + wt) * kStep;
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const int p = p0 + 16 * a;
                const int e = step < step1 && p < end ? entries[p >> c.page_shift] : -1;
                page[a] = __builtin_amdgcn_readfirstlane((uint32_t)e < (uint32_t)c.pages ? e : -1);
            }
        };
        auto offset_of = [&](int step, int a, int page) {
            const int p = (step * kWT + wt) * kStep + 16 * a;
            return head_at + (page < 0 ? 0 : page * c.page_stride + (p & in_page) * c.place_stride);
        };
        uint4 kf[2][kKC];
        auto load_k = [&](int step, const int (&page)[2]) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const char *base = reinterpret_cast<const char *>(c.k + offset_of(step, a, page[a]));
#pragma unroll
                for (int k = 0; k < kKC; ++k)
                    if (EXACT) kf[a][k] = *reinterpret_cast<const uint4 *>(base + koff[0] + 64 * k);
                    else if (32 * k < D) kf[a][k] = *reinterpret_cast<const uint4 *>(base + koff[k]);
            }
        };

        f32x4 o[NQ][kO];
        float m[NQ], l[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            m[x] = kLowest;
            l[x] = 0.f;
#pragma unroll
            for (int j = 0; j < kO; ++j) o[x][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        int page[2], next[2];
        pages_of_step(step0, page);
        pages_of_step(step0 + 1, next);
        load_k(step0, page);
        for (int step = step0; step < step1; ++step) {
            const int p0 = (step * kWT + wt) * kStep;
            if (p0 >= end) break;                                      // (the last step of a tile may have no places for this wavefront)
            // V of this step: pieces of the eight places (tile a, 4 g + i) that the lane's weights are for
            uint32_t vf[8][kHalves * kVW / 2];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const char *base = reinterpret_cast<const char *>(c.v + offset_of(step, a, page[a]));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) {
                        const char *from = base + voff[EXACT ? i : 4 * h + i] + (EXACT ? 256 * h : 0);
                        if constexpr (kVW == 8) {
                            const uint4 x = *reinterpret_cast<const uint4 *>(from);
                            vf[4 * a + i][4 * h] = x.x; vf[4 * a + i][4 * h + 1] = x.y; vf[4 * a + i][4 * h + 2] = x.z; vf[4 * a + i][4 * h + 3] = x.w;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2 *>(from);
                            vf[4 * a + i][0] = x.x; vf[4 * a + i][1] = x.y;
                        }
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            f32x4 sc[NQ][2];
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < kKC; ++k)
                        if (EXACT || 32 * k < D) acc = mma<F16>(kf[a][k], qf[x][k], acc);
                    sc[x][a] = acc;
                }
            __builtin_amdgcn_sched_barrier(0);
            const bool masked = p0 + kStep > len || page[0] < 0 || page[1] < 0;
            const int page0 = page[0], page1 = page[1];
            // the next step's keys while this one's weights are made
            page[0] = next[0]; page[1] = next[1];
            load_k(step + 1, page);
            pages_of_step(step + 2, next);
            __builtin_amdgcn_sched_barrier(0);

            uint32_t seen[NQ];
            uint32_t there = 0xffffffffu;                              // bit n: place p0 + n is one of the sequence's and has a page
            if (masked) {
                const int left = end - p0;
                there = left >= 32 ? 0xffffffffu : (1u << left) - 1;
                if (page0 < 0) there &= 0xffff0000u;
                if (page1 < 0) there &= 0x0000ffffu;
                const int j0 = p0 - len;                               // new token of the step's first place; negative: committed places first
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    // bits of the new tokens j0 .. j0 + 31
                    uint32_t w = 0;
                    if (call.mask) {
                        const int t = row_ok[x] ? row_t[x] : 0;
                        const uint64_t *words = call.mask + (int64_t)(first + t) * call.mask_words;
                        const int w0 = j0 >> 6, sh = j0 & 63;
                        const uint64_t lo = w0 >= 0 && w0 < call.mask_words ? words[w0] : 0;
                        const uint64_t hi = w0 + 1 >= 0 && w0 + 1 < call.mask_words ? words[w0 + 1] : 0;
                        w = (uint32_t)(lo >> sh) | (sh > 32 ? (uint32_t)(hi << (64 - sh)) : 0u);
                    } else {
                        const int k = row_t[x] - j0;                   // the last one that is seen
                        w = k >= 31 ? 0xffffffffu : k >= 0 ? (2u << k) - 1 : 0u;
                    }
                    if (j0 < 0) w |= j0 <= -32 ? 0xffffffffu : (1u << -j0) - 1;
                    seen[x] = w & there;
                }
            }
            uint4 pf[NQ];
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                if (masked) {
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(seen[x] >> (16 * a + 4 * g + i) & 1)) sc[x][a][i] = kNegInf;
                }
                float top = fmaxf(fmaxf(fmaxf(sc[x][0][0], sc[x][0][1]), fmaxf(sc[x][0][2], sc[x][0][3])),
                                  fmaxf(fmaxf(sc[x][1][0], sc[x][1][1]), fmaxf(sc[x][1][2], sc[x][1][3])));
                top = row_max(top) * unit;
                // (unseen everywhere: -infinity, which passes nothing; a scale of 0 makes it not a number, and then 0 is as good a reference)
                const bool moves = top > m[x] + kSlack;
                if (__ballot(moves)) {
                    const float to = moves ? top : m[x], f = __builtin_amdgcn_exp2f(m[x] - to);
                    m[x] = to;
                    l[x] *= f;
#pragma unroll
                    for (int j = 0; j < kO; ++j) o[x][j] *= f;
                }
                float w[8];
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[4 * a + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x][a][i], unit, -m[x]));
                        l[x] += w[4 * a + i];
                    }
                pf[x] = make_uint4(pack2<F16>(w[0], w[1]), pack2<F16>(w[2], w[3]), pack2<F16>(w[4], w[5]), pack2<F16>(w[6], w[7]));
            }
            bool odd_values = false;
            if (masked) {
                // values of places that are nobody's must not meet even a weight of zero; of new tokens, which some rows see and others do
                // not, those that are no numbers or infinite are left out here and added below
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const bool here = there >> (16 * (n >> 2) + 4 * g + (n & 3)) & 1;
#pragma unroll
                    for (int w = 0; w < kHalves * kVW / 2; ++w) {
                        uint32_t v = here ? vf[n][w] : 0u;
                        const bool lo = not_a_number_or_infinite<F16>(v), hi = not_a_number_or_infinite<F16>(v >> 16);
                        odd_values |= lo || hi;
                        v = (lo ? 0u : v & 0x0000ffffu) | (hi ? 0u : v & 0xffff0000u);
                        vf[n][w] = v;
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int j = 0; j < kVW; ++j) {
                    constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;       // (the second operand's halves are bytes 0 to 3)
                    const int w = (kVW / 2) * h + (j >> 1);
                    uint4 a;
                    a.x = __builtin_amdgcn_perm(vf[1][w], vf[0][w], j & 1 ? kHigh : kLow);
                    a.y = __builtin_amdgcn_perm(vf[3][w], vf[2][w], j & 1 ? kHigh : kLow);
                    a.z = __builtin_amdgcn_perm(vf[5][w], vf[4][w], j & 1 ? kHigh : kLow);
                    a.w = __builtin_amdgcn_perm(vf[7][w], vf[6][w], j & 1 ? kHigh : kLow);
#pragma unroll
                    for (int x = 0; x < NQ; ++x) o[x][kVW * h + j] = mma<F16>(a, pf[x], o[x][kVW * h + j]);
                }
            if (masked && __ballot(odd_values)) {
                // rare: the values left out, place by place, to the rows that see the place (whatever its weight: the result is no number or infinite)
                for (int n = 0; n < 32; ++n) {
                    if (!(there >> n & 1)) continue;
                    const int a = n >> 4;
                    const uint16_t *vr = c.v + offset_of(step, a, a ? page1 : page0) + (n & 15) * c.place_stride;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int j = 0; j < kVW; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int d = 128 * h + kVW * (4 * g + i) + j;
                                if (!EXACT && d >= D) continue;
                                const uint16_t v = vr[d];
                                if (!not_a_number_or_infinite<F16>(v)) continue;
#pragma unroll
                                for (int x = 0; x < NQ; ++x)
                                    if (seen[x] >> n & 1) o[x][kVW * h + j][i] += value_of<F16>(v);
                            }
                }
            }
        }

        // the wavefronts of the same rows join: halves to halves, through shared memory in the accumulators' own layout
        if constexpr (kWT > 1) {
            constexpr int kPart = kO * NQ * 256 + 2 * NQ * 64;
#pragma unroll
            for (int half = kWT / 2; half > 0; half >>= 1) {
                float *mine = joint + ((wt % half) * WR + wr) * kPart;
                if (wt >= half && wt < 2 * half) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
#pragma unroll
                        for (int j = 0; j < kO; ++j) *reinterpret_cast<f32x4 *>(mine + ((x * kO + j) * 64 + lane) * 4) = o[x][j];
                        mine[kO * NQ * 256 + (2 * x) * 64 + lane] = m[x];
                        mine[kO * NQ * 256 + (2 * x + 1) * 64 + lane] = l[x];
                    }
                }
                __syncthreads();
                if (wt < half) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
                        const float m2 = mine[kO * NQ * 256 + (2 * x) * 64 + lane], l2 = mine[kO * NQ * 256 + (2 * x + 1) * 64 + lane];
                        const float to = fmaxf(m[x], m2), f = __builtin_amdgcn_exp2f(m[x] - to), f2 = __builtin_amdgcn_exp2f(m2 - to);
                        m[x] = to;
                        l[x] = l[x] * f + l2 * f2;
#pragma unroll
                        for (int j = 0; j < kO; ++j) o[x][j] = o[x][j] * f + *reinterpret_cast<f32x4 *>(mine + ((x * kO + j) * 64 + lane) * 4) * f2;
                    }
                }
                __syncthreads();
            }
        }
        if (wt == 0) {
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const float sum = row_sum(l[x]);
                if (!row_ok[x]) continue;
                if (whole) {
                    // (a row that saw nothing has sums of zero)
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    uint16_t *to = call.out + (int64_t)(first + row_t[x]) * call.out_token_stride + (int64_t)row_h[x] * call.out_head_stride;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int e = 0; e < kVW / 2; ++e) {          // eight adjacent channels of the lane's 4 kVW
                            const int d = 128 * h + 4 * kVW * g + 8 * e;
                            if (!EXACT && d >= D) continue;
                            float y[8];
#pragma unroll
                            for (int n = 0; n < 8; ++n) y[n] = o[x][kVW * h + (8 * e + n) % kVW][(8 * e + n) / kVW] * inv;
                            *reinterpret_cast<uint4 *>(to + d) = make_uint4(pack2<F16>(y[0], y[1]), pack2<F16>(y[2], y[3]), pack2<F16>(y[4], y[5]), pack2<F16>(y[6], y[7]));
                        }
                    if (call.lse && g == 0)
                        call.lse[(int64_t)(first + row_t[x]) * call.q_heads + row_h[x]] = sum == 0.f ? kNegInf : (m[x] + __builtin_amdgcn_logf(sum)) * kLn2;
                } else {
                    float *piece = pieces + (size_t)(2 * blockIdx.x + (first_piece ? 0 : 1)) * piece_floats(Tile::kRows, DP);
                    const int row = (wr * NQ + x) * 16 + r;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int e = 0; e < kVW; ++e) {              // four adjacent channels
                            const int d = 128 * h + 4 * kVW * g + 4 * e;
                            f32x4 y;
#pragma unroll
                            for (int n = 0; n < 4; ++n) y[n] = o[x][kVW * h + (4 * e + n) % kVW][(4 * e + n) / kVW];
                            *reinterpret_cast<f32x4 *>(piece + (size_t)row * DP + d) = y;
                        }
                    if (g == 0) {
                        piece[(size_t)Tile::kRows * DP + row] = m[x];
                        piece[(size_t)Tile::kRows * (DP + 1) + row] = sum;
                    }
                }
            }
        }
        first_piece = false;
        u += step1 - step0;
    }
}

// Joins the pieces of the row tiles that more than one block worked on.  Block (token, key head): the group's rows; a thread takes four channels.
template <bool F16, int DP>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(CacheView c, TreeCall call, BatchView b, Tiling tile, const TreePlan *__restrict__ plan,
                                                              const float *__restrict__ pieces)
{
    __shared__ int found;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    const int token = blockIdx.x, head = blockIdx.y, group = call.q_heads / c.heads;
    for (int i = threadIdx.x; i < b.n; i += kThreads)
        if (b.first[i] <= token && token < b.first[i + 1]) found = i;
    __syncthreads();
    if (found < 0) return;
    const Sequence s = sequence_of(c, b, found);
    if (s.tokens == 0) return;
    Division div{plan->units, plan->blocks};
    const int steps = steps_of(s, tile), tiles = row_tiles(s, group, tile);
    const int64_t base = plan->start[found] + (int64_t)head * tiles * steps;
    const size_t stride = piece_floats(tile.rows, DP);
    for (int e = threadIdx.x; e < group * (DP / 4); e += kThreads) {
        const int gq = e / (DP / 4), d = 4 * (e % (DP / 4));
        const int row = (token - s.first) * group + gq, rt = row / tile.rows, in = row - rt * tile.rows;
        const int64_t u0 = base + (int64_t)rt * steps;
        const int b0 = block_of(div, u0), b1 = block_of(div, u0 + steps - 1);
        if (b0 == b1) continue;
        const float *p0 = pieces + (size_t)(2 * b0 + (run_start(div, b0) == u0 ? 0 : 1)) * stride;
        float m = p0[(size_t)tile.rows * DP + in];
        for (int k = b0 + 1; k <= b1; ++k) m = fmaxf(m, pieces[(size_t)2 * k * stride + (size_t)tile.rows * DP + in]);
        float f = __builtin_amdgcn_exp2f(p0[(size_t)tile.rows * DP + in] - m), sum = p0[(size_t)tile.rows * (DP + 1) + in] * f;
        f32x4 o = *reinterpret_cast<const f32x4 *>(p0 + (size_t)in * DP + d) * f;
#pragma unroll 4
        for (int k = b0 + 1; k <= b1; ++k) {
            const float *p = pieces + (size_t)2 * k * stride;
            f = __builtin_amdgcn_exp2f(p[(size_t)tile.rows * DP + in] - m);
            sum += p[(size_t)tile.rows * (DP + 1) + in] * f;
            o += *reinterpret_cast<const f32x4 *>(p + (size_t)in * DP + d) * f;
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int qh = head * group + gq;
        if (d < c.head_dim)
            *reinterpret_cast<uint2 *>(call.out + (int64_t)token * call.out_token_stride + (int64_t)qh * call.out_head_stride + d) =
                make_uint2(pack2<F16>(o[0] * inv, o[1] * inv), pack2<F16>(o[2] * inv, o[3] * inv));
        if (call.lse && d == 0) call.lse[(int64_t)token * call.q_heads + qh] = sum == 0.f ? kNegInf : (m + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

// ---- the host's side: which tiling, how many blocks
struct Choice { int nq, wr, blocks; };
constexpr int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

Choice choose(int n, int tokens, int group, int head_dim)
{
    const int64_t rows = n > 0 ? (int64_t)((tokens + n - 1) / n) * group : 0;       // of an average sequence's key head
    const bool wide = padded(head_dim) == 256;
    Choice k;
    if (rows <= 16) { k.nq = 1; k.wr = 1; }
    else if (rows <= 32) { k.nq = wide ? 1 : 2; k.wr = wide ? 2 : 1; }
    else if (rows <= 64) { k.nq = wide ? 1 : 2; k.wr = wide ? 4 : 2; }
    else { k.nq = wide ? 1 : 2; k.wr = 4; }
    k.blocks = 256 * (wide || k.nq > 1 ? 2 : 3);
    return k;
}

template <bool F16, int DP, bool EXACT, int NQ, int WR>
hipError_t launch(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, int blocks, TreePlan *plan, float *pieces, hipStream_t st)
{
    using Tile = TileOf<NQ, WR>;
    tree_rows_kernel<F16, DP, EXACT, NQ, WR><<<blocks, kThreads, 0, st>>>(c, layer, call, b, plan, pieces);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    tree_merge_kernel<F16, DP><<<dim3(b.tokens, c.heads), kThreads, 0, st>>>(c, call, b, Tiling{Tile::kRows, Tile::kPlaces}, plan, pieces);
    return hipGetLastError();
}

template <bool F16, int DP, bool EXACT>
hipError_t launch_tiling(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, const Choice &k, TreePlan *plan, float *pieces, hipStream_t st)
{
    if constexpr (DP == 256) {
        if (k.wr == 1) return launch<F16, DP, EXACT, 1, 1>(c, layer, call, b, k.blocks, plan, pieces, st);
        if (k.wr == 2) return launch<F16, DP, EXACT, 1, 2>(c, layer, call, b, k.blocks, plan, pieces, st);
        return launch<F16, DP, EXACT, 1, 4>(c, layer, call, b, k.blocks, plan, pieces, st);
    } else {
        if (k.nq == 1) return launch<F16, DP, EXACT, 1, 1>(c, layer, call, b, k.blocks, plan, pieces, st);
        if (k.wr == 1) return launch<F16, DP, EXACT, 2, 1>(c, layer, call, b, k.blocks, plan, pieces, st);
        if (k.wr == 2) return launch<F16, DP, EXACT, 2, 2>(c, layer, call, b, k.blocks, plan, pieces, st);
        return launch<F16, DP, EXACT, 2, 4>(c, layer, call, b, k.blocks, plan, pieces, st);
    }
}

template <bool F16>
hipError_t launch_type(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, const Choice &k, TreePlan *plan, float *pieces, hipStream_t st)
{
    switch (c.head_dim) {
    case 64: return launch_tiling<F16, 64, true>(c, layer, call, b, k, plan, pieces, st);
    case 128: return launch_tiling<F16, 128, true>(c, layer, call, b, k, plan, pieces, st);
    case 256: return launch_tiling<F16, 256, true>(c, layer, call, b, k, plan, pieces, st);
    }
    if (c.head_dim < 64) return launch_tiling<F16, 64, false>(c, layer, call, b, k, plan, pieces, st);
    if (c.head_dim < 128) return launch_tiling<F16, 128, false>(c, layer, call, b, k, plan, pieces, st);
    return launch_tiling<F16, 256, false>(c, layer, call, b, k, plan, pieces, st);
}

}  // namespace

// The largest that a call of this many or fewer sequences and tokens can need: the widest tiling that so many rows take, all of one sequence.
size_t tree_attention_workspace_bytes(int n, int tokens, int q_heads, int heads, int head_dim)
{
    const int group = q_heads / heads, dp = padded(head_dim);
    size_t floats = 0;
    for (const int rows : {1, 32, 64, 128}) {
        const int t = (int)std::min<int64_t>(tokens, (rows + group - 1) / group);
        const Choice k = choose(1, t, group, head_dim);
        floats = std::max(floats, 2 * (size_t)k.blocks * piece_floats(16 * k.nq * k.wr, dp));
    }
    const Choice k = choose(1, tokens, group, head_dim);
    floats = std::max(floats, 2 * (size_t)k.blocks * piece_floats(16 * k.nq * k.wr, dp));
    return plan_bytes(n) + 4 * floats;
}

hipError_t launch_tree_attention(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, void *workspace, hipStream_t st)
{
    TreePlan *plan = static_cast<TreePlan *>(workspace);
    float *pieces = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan_bytes(b.n));
    const Choice k = choose(b.n, b.tokens, call.q_heads / c.heads, c.head_dim);
    return call.f16 ? launch_type<true>(c, layer, call, b, k, plan, pieces, st) : launch_type<false>(c, layer, call, b, k, plan, pieces, st);
}

}  // namespace slimspec
