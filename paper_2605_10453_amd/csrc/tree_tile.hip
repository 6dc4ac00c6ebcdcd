// Tree attention of many rows to a key head: keys and values go through shared memory.
//
// A block is four wavefronts of 16 NQ query rows each, all on the same 32 places: with as many rows the wavefronts' own loads of K and V
// (tree_rows_kernel) would need several times what a CU's vector cache gives.  The products, their operand orders and the weights are those
// of tree_rows_kernel; V turns on its way out of shared memory (ds_read_b64_tr_b16: 16 lanes read a 4 x 16 block and get its columns).
//
// Stages of 32 places, K and V, come straight into shared memory (global_load_lds_dwordx4), NBUF - 1 ahead, across the pieces of the run.
// A place is DP channels in pieces of 16 bytes, stored at piece index XOR f(place) so that neither a fragment of K (16 places, one piece
// each per lane group) nor one of V meets a bank twice; the loads choose their source accordingly.  Every wavefront issues LPS loads a stage,
// whatever is left to do, and vector memory returns in order: s_waitcnt vmcnt((NBUF - 2) LPS) = its part of the stage needed next has
// landed (other loads and stores only make the wait longer); the barrier then says so for all, and that all have read the stage before.
#include "tree_parts.hpp"
#include <type_traits>

namespace slimspec {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#define LDS_PTR(T, byte_addr) ((__attribute__((address_space(3))) T *)(uintptr_t)(byte_addr))

// 16 bytes per lane, global memory -> LDS at `to` + 16 * lane (uniform)
__device__ __forceinline__ void load_to_lds(uint32_t to, uint32_t voff, const void *base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(to), "v"(voff), "s"(base) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

template <int DP> struct Stage {
    static constexpr int kRow = 2 * DP, kHalf = kStep * kRow, kBytes = 2 * kHalf;      // a place; K; K and V
    static constexpr int kBufs = DP == 256 ? 2 : 4;
    static constexpr int kLoads = kHalf / 1024 / kWaves;                               // per wavefront, for each of K and V
    static constexpr int kWait = (kBufs - 2) * 2 * kLoads;
    static constexpr int kPieces = DP / 8, kPlacesPerLoad = 64 / kPieces;
    static __device__ __forceinline__ int f(int place) { return DP == 64 ? (place >> 1) & 7 : place & 15; }
};

template <bool F16, int DP, bool EXACT, int NQ>
__global__ __launch_bounds__(kThreads, 2) void tree_tile_kernel(TreeArgs args)
{
    using S = Stage<DP>;
    constexpr int kKC = DP / 32, kO = DP / 16, kRows = 64 * NQ;
    __shared__ __align__(1024) unsigned char stages[S::kBufs * S::kBytes];
    __shared__ int4 near[kNear];
    __shared__ int odd_in;                                             // the last masked step (counted from 1) with values left out
    const CacheView &c = args.c;
    const TreeCall &call = args.call;
    const BatchView &b = args.b;
    const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)stages);
    const Tiling tile{kRows, kStep};
    const int group = call.q_heads / c.heads;
    Division div;
    Run run = divide<kWaves>(c, b, group, tile, div, args.plan, near);
    if (run.u >= run.end) return;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int D = EXACT ? DP : c.head_dim;
    const int in_page = (1 << c.page_shift) - 1;
    const float scaled = call.scale * kLog2e, unit = fabsf(scaled) >= 1.2e-38f ? scaled : 1.2e-38f;    // (not 0: an unseen place's infinite score stays one)

    // ---- loading: this lane's source offsets from the first of 16 places (pieces past head_dim: the place's first one again)
    uint32_t voff[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const int place = (wave * S::kLoads + i) * S::kPlacesPerLoad + lane / S::kPieces, piece = (lane % S::kPieces) ^ S::f(place);
        voff[i] = (uint32_t)(place & 15) * 2u * (uint32_t)c.place_stride + (EXACT || 8 * piece < D ? 16u * piece : 0u);
    }
    Run ahead = run;
    Piece lp = next_piece(c, b, group, tile, near, ahead);
    int lstep = lp.step0, page[2];
    bool lmore = true;                                                 // stages left to load
    uint32_t no_pages = 0;                                             // two bits per stage issued, the latest lowest: its stretches of 16 without a page
    auto pages_of_step = [&]() {
        const auto *entries = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(c.table + (int64_t)lp.slot * c.slot_pages);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int place = lstep * kStep + 16 * a;
            const int e = lmore && place < lp.len + lp.tokens ? entries[place >> c.page_shift] : -1;
            page[a] = __builtin_amdgcn_readfirstlane((uint32_t)e < (uint32_t)c.pages ? e : -1);
        }
    };
    auto issue = [&](uint32_t buf) {
        int64_t at[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int place = lstep * kStep + 16 * a;
            at[a] = lp.head * c.head_stride + (page[a] < 0 ? 0 : page[a] * c.page_stride + (place & in_page) * c.place_stride);
        }
        no_pages = no_pages << 2 | (page[0] < 0 ? 1u : 0u) | (page[1] < 0 ? 2u : 0u);
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const int n = wave * S::kLoads + i;
            const int64_t from = n * S::kPlacesPerLoad >= 16 ? at[1] : at[0];
            load_to_lds(buf + n * 1024, voff[i], c.k + from);
            load_to_lds(buf + S::kHalf + n * 1024, voff[i], c.v + from);
        }
        if (lmore && ++lstep == lp.step1) {
            lmore = ahead.u < ahead.end;
            if (lmore) {
                lp = next_piece(c, b, group, tile, near, ahead);
                lstep = lp.step0;
            }
        }
        pages_of_step();
    };

    // ---- reading: K's fragment (a, k) at (buf + ka) ^ (k << 6), 16 a places on; V's (j, half) at (buf + va) ^ (j << 5), 16 places on
    const uint32_t ka = r * S::kRow + ((g ^ S::f(r)) << 4);
    const int vplace = 4 * g + (r >> 2);
    const uint32_t va = S::kHalf + vplace * S::kRow + ((((r >> 1) & 1) ^ S::f(vplace)) << 4) + ((r & 1) << 3);

    // ---- this lane's query rows: number x in a piece is token t of the sequence and query head h
    uint4 qf[NQ][kKC];
    auto row_of = [&](const Piece &p, int x, int &t, int &h) {
        const int row = p.rt * kRows + (wave * NQ + x) * 16 + r;
        t = row / group;
        h = p.head * group + row - t * group;
        return t < p.tokens;
    };
    auto load_q = [&](const Piece &p) {
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            int t, h;
            const bool ok = row_of(p, x, t, h);
            const uint16_t *qr = call.q + (int64_t)(p.first + (ok ? t : 0)) * call.q_token_stride + (int64_t)(ok ? h : 0) * call.q_head_stride;
#pragma unroll
            for (int k = 0; k < kKC; ++k) {
                qf[x][k] = make_uint4(0, 0, 0, 0);
                if (ok && (EXACT || 32 * k + 8 * g < D)) qf[x][k] = *reinterpret_cast<const uint4 *>(qr + 32 * k + 8 * g);
            }
        }
    };
    // Rows' references: ref, minus the reference as the accumulators start from it, in units of raw scores (four times the same: an operand of the
    // first product); the reference is 0 until the row's first score, and slack says so (kLowest, then kSlack)
    f32x4 o[NQ][kO], ref[NQ];
    float slack[NQ], l[NQ];
    auto clear = [&]() {
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            ref[x] = (f32x4){0.f, 0.f, 0.f, 0.f};
            slack[x] = kLowest;
            l[x] = 0.f;
#pragma unroll
            for (int j = 0; j < kO; ++j) o[x][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
    };

    pages_of_step();
    uint32_t buf = lds0, buf_ahead = lds0;
    auto next_buf = [&](uint32_t x) { return x + S::kBytes == lds0 + S::kBufs * S::kBytes ? lds0 : x + S::kBytes; };
#pragma unroll
    for (int s = 0; s < S::kBufs - 1; ++s) {
        issue(buf_ahead);
        buf_ahead = next_buf(buf_ahead);
    }
    Piece p = next_piece(c, b, group, tile, near, run);
    load_q(p);
    clear();
    bool first_piece = true;
    int step = p.step0, masked_steps = 0;
    if (threadIdx.x == 0) odd_in = 0;
    while (true) {
        wait_loads<S::kWait>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        issue(buf_ahead);
        buf_ahead = next_buf(buf_ahead);

        const int p0 = step * kStep, end = p.len + p.tokens;
        const uint32_t no_page = no_pages >> 2 * (S::kBufs - 1) & 3;
        const bool masked = p0 + kStep > p.len || no_page;
        const uint32_t there = masked ? places_there(p0, end, no_page) : 0xffffffffu;
        bool odd_values = false;
        if (masked) {
            // The block's wavefronts rid the stage's values of what must not meet even a weight of zero: places that are nobody's; and of new
            // tokens, which some rows see and others do not, values that are no numbers or infinite, which are added below to the rows that see them.
            ++masked_steps;
            bool odd = false;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i) {
                const int n = wave * S::kLoads + i, place = n * S::kPlacesPerLoad + lane / S::kPieces;
                const auto at = LDS_PTR(u32x4, buf + S::kHalf + n * 1024 + 16 * lane);
                u32x4 v = *at;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t x = v[w];
                    odd |= leave_out<F16>(x, there >> place & 1);
                    v[w] = x;
                }
                *at = v;
            }
            if (__ballot(odd) && lane == 0) odd_in = masked_steps;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            odd_values = __builtin_amdgcn_readfirstlane(*(volatile int *)&odd_in) == masked_steps;
        }
        f32x4 sc[NQ][2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            u32x4 kf[kKC];
#pragma unroll
            for (int k = 0; k < kKC; ++k)
                if (EXACT || 32 * k < D) kf[k] = *LDS_PTR(u32x4, ((buf + ka) ^ (k << 6)) + 16 * a * S::kRow);
#pragma unroll
            for (int x = 0; x < NQ; ++x) sc[x][a] = ref[x];
#pragma unroll
            for (int k = 0; k < kKC; ++k)
                if (EXACT || 32 * k < D)
#pragma unroll
                    for (int x = 0; x < NQ; ++x) sc[x][a] = mma<F16>(__builtin_bit_cast(uint4, kf[k]), qf[x][k], sc[x][a]);
        }
        uint32_t seen[NQ];
        if (masked) {
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                int t, h;
                seen[x] = places_seen(call, p.first, row_of(p, x, t, h) ? t : 0, p0 - p.len, there);
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(seen[x] >> (16 * a + 4 * g + i) & 1)) sc[x][a][i] = unit < 0.f ? -kNegInf : kNegInf;
            }
        }
        // scores in bits, relative to the references; where one passes its reference by too much, or a row has its first, sums are scaled
        float top[NQ];
        bool moves = false;
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            sc[x][0] *= unit;
            sc[x][1] *= unit;
            top[x] = row_max(fmaxf(fmaxf(fmaxf(sc[x][0][0], sc[x][0][1]), fmaxf(sc[x][0][2], sc[x][0][3])),
                                   fmaxf(fmaxf(sc[x][1][0], sc[x][1][1]), fmaxf(sc[x][1][2], sc[x][1][3]))));
            moves |= top[x] > slack[x];
        }
        if (__ballot(moves)) {
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const bool first_one = slack[x] == kLowest;
                const float by = top[x] > slack[x] ? top[x] : 0.f, f = first_one ? 0.f : __builtin_amdgcn_exp2f(-by);
                if (top[x] > slack[x]) slack[x] = kSlack;
                const float raw = ref[x][0] - by / unit;
                ref[x] = (f32x4){raw, raw, raw, raw};
                l[x] *= f;
                sc[x][0] -= by;
                sc[x][1] -= by;
#pragma unroll
                for (int j = 0; j < kO; ++j) o[x][j] *= f;
            }
        }
        uint4 pf[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            float w[8];
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) w[4 * a + i] = __builtin_amdgcn_exp2f(sc[x][a][i]);
            l[x] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            pf[x] = make_uint4(pack2<F16>(w[0], w[1]), pack2<F16>(w[2], w[3]), pack2<F16>(w[4], w[5]), pack2<F16>(w[6], w[7]));
        }
#pragma unroll
        for (int j = 0; j < kO; ++j) {
            const uint32_t at = (buf + va) ^ (j << 5);
            const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(i16x4, at)));
            const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(i16x4, at + 16 * S::kRow)));
            const uint4 v = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int x = 0; x < NQ; ++x) o[x][j] = mma<F16>(v, pf[x], o[x][j]);
        }
        if (odd_values) {
            // rare: the values left out, place by place, to the rows that see the place (whatever its weight: the result is no number or infinite)
            for (int n = 0; n < 32; ++n) {
                if (!(there >> n & 1)) continue;
                const int place = p0 + n, of = page_of(c, p.slot, place);
                const uint16_t *vr = c.v + p.head * c.head_stride + of * c.page_stride + (place & in_page) * c.place_stride;
#pragma unroll
                for (int j = 0; j < kO; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = 16 * j + 4 * g + i;
                        if (!EXACT && d >= D) continue;
                        const uint16_t v = vr[d];
                        if (!not_a_number_or_infinite<F16>(v)) continue;
#pragma unroll
                        for (int x = 0; x < NQ; ++x)
                            if (seen[x] >> n & 1) o[x][j][i] += value_of<F16>(v);
                    }
            }
        }
        buf = next_buf(buf);
        if (++step < p.step1) continue;

#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            const float sum = row_sum(l[x]), m = slack[x] == kLowest ? kLowest : -ref[x][0] * unit;
            int t, h;
            if (!row_of(p, x, t, h)) continue;
            if (p.whole) {
                const float inv = inverse(sum);
                uint16_t *to = call.out + (int64_t)(p.first + t) * call.out_token_stride + (int64_t)h * call.out_head_stride + 4 * g;
#pragma unroll
                for (int j = 0; j < kO; ++j)
                    if (EXACT || 16 * j + 4 * g < D)
                        *reinterpret_cast<uint2 *>(to + 16 * j) = make_uint2(pack2<F16>(o[x][j][0] * inv, o[x][j][1] * inv), pack2<F16>(o[x][j][2] * inv, o[x][j][3] * inv));
                if (call.lse && g == 0) call.lse[(int64_t)(p.first + t) * call.q_heads + h] = lse_of(m, sum);
            } else {
                float *piece = args.pieces + (size_t)(2 * run.block + (first_piece ? 0 : 1)) * piece_floats(kRows, DP);
                const int row = (wave * NQ + x) * 16 + r;
#pragma unroll
                for (int j = 0; j < kO; ++j) *reinterpret_cast<f32x4 *>(piece + (size_t)row * DP + 16 * j + 4 * g) = o[x][j];
                if (g == 0) {
                    piece[(size_t)kRows * DP + row] = m;
                    piece[(size_t)kRows * (DP + 1) + row] = sum;
                }
            }
        }
        if (run.u >= run.end) break;
        first_piece = false;
        p = next_piece(c, b, group, tile, near, run);
        step = p.step0;
        load_q(p);
        clear();
    }
    wait_loads<0>();                                                   // no load into the block's shared memory outlives the block
}

template <bool F16, int DP, bool EXACT>
hipError_t launch_nq(const TreeArgs &a, int nq, int blocks, hipStream_t st)
{
    if constexpr (DP == 64) tree_tile_kernel<F16, DP, EXACT, 4><<<blocks, kThreads, 0, st>>>(a);
    else if constexpr (DP == 128) tree_tile_kernel<F16, DP, EXACT, 3><<<blocks, kThreads, 0, st>>>(a);
    else tree_tile_kernel<F16, DP, EXACT, 1><<<blocks, kThreads, 0, st>>>(a);
    return hipGetLastError();
}
template <bool F16>
hipError_t launch_type(const TreeArgs &a, int nq, int blocks, hipStream_t st)
{
    const int d = a.c.head_dim;
    if (d <= 64) return d == 64 ? launch_nq<F16, 64, true>(a, nq, blocks, st) : launch_nq<F16, 64, false>(a, nq, blocks, st);
    if (d <= 128) return d == 128 ? launch_nq<F16, 128, true>(a, nq, blocks, st) : launch_nq<F16, 128, false>(a, nq, blocks, st);
    return d == 256 ? launch_nq<F16, 256, true>(a, nq, blocks, st) : launch_nq<F16, 256, false>(a, nq, blocks, st);
}

}  // namespace

hipError_t launch_tree_tile(const TreeArgs &a, int nq, int blocks, hipStream_t st)
{
    return a.call.f16 ? launch_type<true>(a, nq, blocks, st) : launch_type<false>(a, nq, blocks, st);
}

}  // namespace slimspec
