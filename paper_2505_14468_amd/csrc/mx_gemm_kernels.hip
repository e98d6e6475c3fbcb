// Tiled product of a 4-bit backbone and 8-bit activations, both with a scale for every 32 values, with the LoRA expand behind it:
//
//     Y[row, n] = sum_k X[row, k] W[n, k]  +  sum_j V[row, j] B_a[n, j]  (+ D[row, n]),   row = perm[slot], rounded once
//
// The base product runs on the block-scaled matrix instructions: one 16x16x128 MFMA takes 128 values of 16 rows of W (e2m1) and of
// 16 rows of X (e4m3) with the scales of their blocks, so nothing is ever taken apart.  Of a 16-row operand of W, lane l holds
// block l / 16 of row l % 16 (16 bytes); of X the 16-byte pieces l / 16 and 4 + l / 16 of the row's 128 bytes (measured: element e
// of lane group g is value 16 g + e for e < 16, 48 + 16 g + e behind); the scale operand is that of block l / 16 for both, one byte
// of a register that holds four.
//
// Activations of PARTS == 2 come as the sum of two sets of 8-bit values (a bf16 row taken apart, mx_split_kernel): the
// contraction axis is walked twice, once for each, against the same W.
//
// Tile: BM rows x BN columns, stages of 128 values of the contraction axis, D of them in LDS, loaded there directly.  4
// waves, one per SIMD, each a quarter of the tile.  What a stage costs a wave besides its MFMAs (256 x 256: 64 of them, 32
// cycles each) is 24 operand reads, 12 loads and a few scalar instructions, dealt out one behind an MFMA; the scales cost
// next to nothing: they are loaded, put into the order that the instruction wants and read once for four stages together.
//
// The wave's tile is cut into halves along both sides, W0 W1 and X0 X1; a stage multiplies its four quadrants in the order
//     (W0, Xa) (W0, Xb) | barrier | (W1, Xb) (W1, Xa)         a = 0, b = 1 in even stages, the reverse in odd ones
// so that every half of the operands is free a quadrant before the next stage's takes its registers: Xb and W1 are read from LDS
// during the first quadrant, W0 of the next stage during the third, its first X half (this one's Xb) during the fourth.
// The one barrier of a stage therefore stands where all of the stage has been read: its LDS takes stage kt + D at once, which then has
// D - 1 stages to arrive.  256 x 256: D = 2 (a stage is 2048 cycles of MFMAs); 128 x 256 and 128 x 128, whose stages are a half and a
// quarter of that, D = 4.
//
// The extension is more stages of the same pipeline, of 32 ranks each, on bf16 16x16x32 MFMAs: the rows of a tile are in slot order, so
// an adapter's are contiguous, and its V and B_a take the places of X and W in LDS (rows of B_a of 64 bytes are laid out as W's,
// rows of V as the first halves of X's).  The first are requested where the base product has nothing left to request.
// Rows of other adapters and ranks past the adapter's own are loads out of the descriptor's range: zeros that cost no
// traffic.  A tile's segments are found by one thread each and kept in a table.
#include <type_traits>
#include <utility>

#include "mx_common.hiph"

namespace lora {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

template <int A, typename F, int... I>
__device__ __forceinline__ void for_impl(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, A + I>{}), ...);
}
template <int A, int B, typename F>
__device__ __forceinline__ void for_each(F &&f) {
    for_impl<A>(f, std::make_integer_sequence<int, (B > A ? B - A : 0)>{});
}

// LDS position (in 16-byte pieces) of piece c of row r: rows of X of 8 pieces, rows of W of 4, two to a line of 8.  16 rows of one
// piece column, as an operand read takes them, then lie in 16 different quarters of the banks.
__device__ __forceinline__ int x_at(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }
__device__ __forceinline__ int w_at(int r, int c) { return (r >> 1) * 8 + ((((r & 1) << 2) | c) ^ mx_quarter((r >> 2) & 3)); }

// acc += W X on byte S of the scale registers, in place.  Assembly for the reason that Elem<>::mma_step gives: the accumulators
// stay in their registers; mma_settle keeps the distance to whatever touches them next.
template <int S>
__device__ __forceinline__ void mma_scaled(f32x4_t &acc, const u32x4_t &w, const i32x8_t &x, unsigned ws, unsigned xs) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (S == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4" : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
    else if constexpr (S == 1)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4" : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
    else if constexpr (S == 2)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0] cbsz:4" : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0] cbsz:4" : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
#else
    (void)acc, (void)w, (void)x, (void)ws, (void)xs;
#endif
}

// A direct load whose descriptor or offset a vector instruction may just have written (a lane read into a scalar register, which is also
// how the compiler brings back scalars it had no room for): 5 wait states, which it keeps in front of its own loads only.  The
// loads of a stage do without: they are a quadrant away from the scalars they use, which is checked in the built code.
__device__ __forceinline__ void load_to_lds_settled(const BufferDesc &d, unsigned lane_off, int scalar_off) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(lane_off), "s"(d.r), "s"(scalar_off));
#else
    (void)d, (void)lane_off, (void)scalar_off;
#endif
}

template <int BM, int BN>
struct MxTile {
    static constexpr int NT = 256, WTM = BM / 2, WTN = BN / 2, NBT = WTM / 16, NBN = WTN / 16, HT = NBT / 2, HN = NBN / 2;
    static constexpr int GX = BM / 32, GW = BN / 64;  // direct loads of a stage per wave
    static constexpr int D = BM * BN >= 65536 ? 2 : 4;  // stages in LDS
    static constexpr size_t x_bytes = (size_t)BM * 128, w_bytes = (size_t)BN * 64, s_bytes = (size_t)(BM + BN) * 16;
    static constexpr size_t smem = D * (x_bytes + w_bytes) + 3 * s_bytes + (size_t)BM * (16 + 4 + 1) + 16;
    static_assert(smem <= 160 * 1024, "LDS of a CU");
    static_assert(NBT % 2 == 0 && NBN % 2 == 0 && HT >= 1 && HN >= 1 && GX >= 1 && GW >= 1 && BM + BN <= 2 * NT && BM <= NT && BN <= NT, "tile shape");
};

// One tile: rows from m0 on (in slot order), column tile pn of all projections'.
template <int BM, int BN, int PARTS, bool SPLIT>
__device__ __forceinline__ void mx_gemm_tile(const MxGemmArgs &p, int m0, int pn) {
    typedef MxTile<BM, BN> M;
    typedef __bf16 E;
    constexpr int NBT = M::NBT, NBN = M::NBN, HT = M::HT, HN = M::HN, GX = M::GX, GW = M::GW, D = M::D;

    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    chunk_t *sX = reinterpret_cast<chunk_t *>(smem);                             // [D][BM * 8]
    chunk_t *sW = reinterpret_cast<chunk_t *>(smem + D * M::x_bytes);            // [D][BN * 4]
    chunk_t *sraw = sW + D * BN * 4;                                             // [BM + BN]: the next superstage's scales as they lie in memory
    chunk_t *sS = sraw + (BM + BN);                                              // [2][BM + BN]: two superstages' in order
    chunk_t *sseg = sS + 2 * (BM + BN);                                          // the tile's segments whose term is computed here
    int *srow = reinterpret_cast<int *>(sseg + BM);                              // tile row -> original row
    int *scnt = srow + BM;                                                       // segments found per wave
    unsigned char *use_d = reinterpret_cast<unsigned char *>(scnt + 4);          // tile row takes its adapter term from D

    int si = 0;
    while (si + 1 < p.n_sets && pn >= p.set[si + 1].tile0) ++si;
    const MxGemmSet g = p.set[si];
    const int n0 = (pn - g.tile0) * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn0 = (wave & 1) * M::WTN, wm0 = (wave >> 1) * M::WTM;
    const int lr = lane & 15, lq = lane >> 4;

    // this workgroup's stretch of the contraction axis, in blocks of 32 and stages of four
    const int nblocks = p.K / kMxBlock;
    int b0 = 0, nloc = nblocks;
    if constexpr (SPLIT) {
        b0 = (int)blockIdx.y * p.chunk_blocks;
        nloc = min(nblocks - b0, p.chunk_blocks);
    }
    // Stages of one part.  (Two parts: whole superstages -- the rows of X are that long and hold zeros past K.)
    const int KP = PARTS == 2 ? (nloc + 15) >> 4 << 2 : (nloc + 3) >> 2;
    const int KT = KP * PARTS;

    // ---- what is loaded where -------------------------------------------------------------------------------------
    const int rx0 = wave * GX * 8, rw0 = wave * GW * 16;  // first tile row of the wave's loads
    int orig[GX];
#pragma unroll
    for (int i = 0; i < GX; ++i) orig[i] = p.plan.perm[min(m0 + rx0 + i * 8 + (lane >> 3), p.T - 1)];
    const int my_row = p.plan.perm[min(m0 + tid % BM, p.T - 1)];
    const int status = p.plan.scalars[kScStatus];
#pragma unroll
    for (int i = 0; i < GX; ++i) asm volatile("" ::"v"(orig[i]));
    if (status != 0) return;  // (a plan that was not built: its rows are whatever the buffer holds)
    if (tid < BM) srow[tid] = my_row;
    // 32-bit byte offsets, X's from its start, W's from the tile's first row; both descriptors end with the last row's last block
    unsigned ox[GX], ow[GW];
#pragma unroll
    for (int i = 0; i < GX; ++i) {
        const int row = rx0 + i * 8 + (lane >> 3);
        ox[i] = (unsigned)((int64_t)orig[i] * p.ldxq) + (unsigned)((lane & 7) ^ ((row >> 1) & 7)) * 16u;
    }
#pragma unroll
    for (int i = 0; i < GW; ++i) {
        const int row = rw0 + i * 16 + 2 * (lane >> 3) + ((lane & 7) >> 2);
        ow[i] = (unsigned)((int64_t)(min(n0 + row, g.N - 1) - n0) * g.ldwq) + (unsigned)((lane & 3) ^ mx_quarter((row >> 2) & 3)) * 16u;
    }
    const unsigned char *Xb = p.Xq + (int64_t)b0 * 32, *Wb = g.Wq + (int64_t)n0 * g.ldwq + b0 * 16;
    const int64_t x_row = PARTS == 2 ? 2 * (int64_t)p.part_bytes : (int64_t)nblocks * 32;  // bytes of a row of X in use
    const int x_range = (int)(unsigned)((int64_t)(p.T - 1) * p.ldxq + x_row - (int64_t)b0 * 32);
    const int w_range = (int)(unsigned)((int64_t)(min(BN, g.N - n0) - 1) * g.ldwq + (int64_t)(nblocks - b0) * 16);
    const unsigned dx = lds_address(sX) + rx0 * 128, dw = lds_address(sW) + rw0 * 64;
    BufferDesc Xd, Wd;
    int x_so = 0, w_so = 0;
    // (loads past the last stage are issued all the same, against descriptors of no bytes)
    auto stage_desc = [&](int kt) __attribute__((always_inline)) {
        int live;
        asm("s_sub_i32 %0, %1, %2\n\ts_ashr_i32 %0, %0, 31" : "=s"(live) : "s"(kt), "s"(KT) : "scc");
        Xd = make_buffer_desc(Xb, x_range & live);
        Wd = make_buffer_desc(Wb, w_range & live);
        if constexpr (PARTS == 1) {
            x_so = __builtin_amdgcn_readfirstlane(kt * 128);
            w_so = __builtin_amdgcn_readfirstlane(kt * 64);
        } else {
            const int part = kt >= KP ? 1 : 0, k = kt - (part ? KP : 0);
            x_so = __builtin_amdgcn_readfirstlane(part * p.part_bytes + k * 128);
            w_so = __builtin_amdgcn_readfirstlane(k * 64);
        }
    };
    auto load_base = [&](auto jc, int buf) __attribute__((always_inline)) {
        constexpr int j = jc.value;
        if constexpr (j < GX)
            set_lds_base<j * 1024>(dx + buf * (int)M::x_bytes);
        else
            set_lds_base<(j - GX) * 1024>(dw + buf * (int)M::w_bytes);
    };
    auto load = [&](auto jc) __attribute__((always_inline)) {
        constexpr int j = jc.value;
        if constexpr (j < GX)
            load_to_lds(Xd, ox[j], x_so);
        else
            load_to_lds(Wd, ow[j - GX], w_so);
    };
    auto load_settled = [&](auto jc) __attribute__((always_inline)) {
        constexpr int j = jc.value;
        if constexpr (j < GX)
            load_to_lds_settled(Xd, ox[j], x_so);
        else
            load_to_lds_settled(Wd, ow[j - GX], w_so);
    };
    // ---- scales, a superstage (four stages) at a time: thread t takes rows t of X's and of W's tile (those of a smaller tile are loaded
    // twice).  Whole superstages are loaded straight into LDS, in front of a stage's loads and like them unknown to the
    // compiler, which would wait for everything in flight with them; a last, partial one through registers, masked. ------------
    const int SP = (KP + 3) >> 2;  // superstages of a part
    const int xs_range = (int)(unsigned)((int64_t)p.T * p.ldxs - b0), ws_range = (int)(unsigned)((int64_t)min(BN, g.N - n0) * g.ldws - b0);
    const BufferDesc Xsd = make_buffer_desc(p.Xs + b0, xs_range), Wsd = make_buffer_desc(g.Ws + (int64_t)n0 * g.ldws + b0, ws_range);
    const unsigned oxs = (unsigned)((int64_t)my_row * p.ldxs), ows = (unsigned)((int64_t)(min(n0 + tid % BN, g.N - 1) - n0) * g.ldws);
    const unsigned dxs = lds_address(sraw) + (unsigned)(wave % (BM / 64)) * 1024u, dws = lds_address(sraw) + (unsigned)(BM * 16 + wave % (BN / 64) * 1024);
    chunk_t xs_new = zero_chunk(), ws_new = zero_chunk();
    auto request_scales = [&](int s) __attribute__((always_inline)) {
        const int part = PARTS == 2 && s >= SP ? 1 : 0, k = s - (part ? SP : 0);
        const int xo = __builtin_amdgcn_readfirstlane(part * p.part_scales + k * 16), wo = __builtin_amdgcn_readfirstlane(k * 16);
        if (k * 16 + 16 <= nloc) {
            set_lds_base<0>(dxs), load_to_lds_settled(Xsd, oxs, xo);
            set_lds_base<0>(dws), load_to_lds_settled(Wsd, ows, wo);
        } else {
            xs_new = mx_load_scales(p.Xs + b0 + (int64_t)my_row * p.ldxs + part * p.part_scales, k, nloc);
            ws_new = mx_load_scales(g.Ws + b0 + (int64_t)min(n0 + tid % BN, g.N - 1) * g.ldws, k, nloc);
        }
    };
    auto order_scales = [&](int s) __attribute__((always_inline)) {
        chunk_t *to = sS + (s & 1) * (BM + BN);
        const int k = PARTS == 2 && s >= SP ? s - SP : s;
        if (k * 16 + 16 <= nloc) {
#pragma unroll
            for (int i = 0; i < (BM + BN + 255) / 256; ++i)
                if ((BM + BN) % 256 == 0 || tid + i * 256 < BM + BN) to[tid + i * 256] = mx_transpose_scales(sraw[tid + i * 256]);
        } else {
            if (tid < BM) to[tid] = mx_transpose_scales(xs_new);
            if (tid < BN) to[BM + tid] = mx_transpose_scales(ws_new);
        }
    };
    request_scales(0);
    // (the base product's first stages are on their way before the segments are looked up: a chain of three dependent reads)
    for_each<0, D>([&](auto sc) __attribute__((always_inline)) {
        if (sc.value < KT) {
            stage_desc(sc.value);
            for_each<0, GX + GW>([&](auto jc) __attribute__((always_inline)) { load_base(jc, sc.value), load_settled(jc); });
        }
    });

    // ---- the tile's segments: those whose term is computed here, and which rows take theirs from D ------------------------------
    int n_seg = 0;
    if (!SPLIT && (g.B != nullptr || g.D != nullptr)) {
        const int m_last = min(m0 + BM, p.T) - 1;
        const int s_first = p.plan.row_seg[m0], s_last = p.plan.row_seg[m_last];
        if (g.D != nullptr && tid < BM) {
            const int s = p.plan.row_seg[min(m0 + tid, m_last)];
            const bool lng = g.long_rows > 0 && p.plan.seg_indptr[s + 1] - p.plan.seg_indptr[s] >= g.long_rows;
            use_d[tid] = p.plan.seg_adapter[s] >= 0 && !lng;
        }
        if (g.B != nullptr) {  // (at most BM of them: each has a row here)
            const int s = s_first + tid;
            int lo = 0, hi = 0, r = 0;
            const void *Ba = nullptr;
            if (s <= s_last && tid < BM) {
                const int ad = p.plan.seg_adapter[s];
                lo = p.plan.seg_indptr[s], hi = p.plan.seg_indptr[s + 1], r = p.plan.seg_rank[s];
                if (ad >= 0 && r > 0 && hi - lo >= g.long_rows) {
                    Ba = g.B[ad];
                    if (Ba == nullptr) atomicMin(&p.plan.scalars[kScEvicted], kErrNotResident);  // slot emptied after the plan
                }
            }
            const unsigned long long found = __builtin_amdgcn_ballot_w64(Ba != nullptr);
            if (lane == 0) scnt[wave] = __builtin_popcountll(found);
            __syncthreads();
            int at = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                at += w < wave ? scnt[w] : 0;
                n_seg += scnt[w];
            }
            at += __builtin_popcountll(found & ((1ull << lane) - 1ull));
            const uint64_t addr = reinterpret_cast<uint64_t>(Ba);
            if (Ba != nullptr) sseg[at] = make_uint4((unsigned)addr, (unsigned)(addr >> 32), (unsigned)r, (unsigned)max(lo - m0, 0) | (unsigned)min(hi - m0, BM) << 16);
            __syncthreads();
            n_seg = __builtin_amdgcn_readfirstlane(n_seg);
        }
    }
    // The next extension stage: 32 ranks of a segment.  span: its tile rows, first | end << 16; 0: there is none.
    int ext_seg = 0, ext_j = 0;
    auto extension_desc = [&]() __attribute__((always_inline)) -> int {
        if (ext_seg >= n_seg) {
            Xd = make_buffer_desc(p.Xq, 0);
            Wd = make_buffer_desc(p.Xq, 0);
            return 0;
        }
        const chunk_t e = sseg[ext_seg];
        const uint64_t addr = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)e.y) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)e.x);
        const int r = __builtin_amdgcn_readfirstlane((int)e.z), span = __builtin_amdgcn_readfirstlane((int)e.w);
        const int lo = span & 0xffff, hi = span >> 16, j0 = ext_j;
        ext_j += 32;
        if (ext_j >= r) ext_j = 0, ++ext_seg;
        x_so = w_so = 0;
        Xd = make_buffer_desc(g.V, (int)(unsigned)((int64_t)p.T * p.r_max * 2));
        Wd = make_buffer_desc(reinterpret_cast<const E *>(addr) + (int64_t)n0 * r, min(BN, g.N - n0) * r * 2);
#pragma unroll
        for (int i = 0; i < GX; ++i) {
            const int row = rx0 + i * 8 + (lane >> 3), j = j0 + ((lane & 7) ^ ((row >> 1) & 7)) * 8;
            ox[i] = row >= lo && row < hi && j < min(j0 + 32, r) ? (unsigned)srow[row] * (unsigned)(p.r_max * 2) + (unsigned)j * 2u : ~15u;
        }
#pragma unroll
        for (int i = 0; i < GW; ++i) {
            const int row = rw0 + i * 16 + 2 * (lane >> 3) + ((lane & 7) >> 2), j = j0 + ((lane & 3) ^ mx_quarter((row >> 2) & 3)) * 8;
            ow[i] = j < r ? (unsigned)(min(n0 + row, g.N - 1) - n0) * (unsigned)(r * 2) + (unsigned)j * 2u : ~15u;
        }
        return span;
    };
    int span[D] = {};  // of the extension stages requested last, the oldest first
    auto next_desc = [&](int kt) __attribute__((always_inline)) {
        if (SPLIT || kt < KT || n_seg == 0) {
            stage_desc(kt);
        } else {
#pragma unroll
            for (int i = 0; i + 1 < D; ++i) span[i] = span[i + 1];
            span[D - 1] = extension_desc();
        }
    };
    __syncthreads();  // (srow)
    for_each<1, D>([&](auto sc) __attribute__((always_inline)) {
        if (sc.value >= KT) {
            next_desc(sc.value);
            for_each<0, GX + GW>([&](auto jc) __attribute__((always_inline)) { load_base(jc, sc.value), load_settled(jc); });
        }
    });

    f32x4_t acc[NBN][NBT];
#pragma unroll
    for (int nb = 0; nb < NBN; ++nb)
#pragma unroll
        for (int tb = 0; tb < NBT; ++tb) acc[nb][tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto settle = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NBN; ++nb) mma_settle(acc[nb]);
    };
    settle();

    // What lies past K in the last stage of a part, once it is there: zeros in X (its codes are other bytes of memory, which may
    // mean NaN; W's always mean something finite, and its scales are zeros there, 2^-127).
    const int tail = PARTS == 1 ? nloc & 3 : 0;
    auto zero_tail = [&](int buf) __attribute__((always_inline)) {
        for (int i = tid; i < BM * 8; i += 256)
            if ((i & 7) >= 2 * tail) sX[buf * BM * 8 + x_at(i >> 3, i & 7)] = zero_chunk();
        __syncthreads();
    };
    auto is_tail = [&](int kt) { return tail != 0 && kt == KT - 1; };

    // ---- base product ---------------------------------------------------------------------------------------------------
    {
        u32x4_t w[2][HN];
        i32x8_t x[2][HT];
        unsigned wsc[2][HN], xsc[2][HT];
        const chunk_t *px0 = sX + x_at(wm0 + lr, lq), *px1 = sX + x_at(wm0 + lr, 4 + lq), *pw = sW + w_at(wn0 + lr, lq);
        const unsigned *psx = reinterpret_cast<const unsigned *>(sS) + (wm0 + lr) * 4 + lq, *psw = reinterpret_cast<const unsigned *>(sS) + (BM + wn0 + lr) * 4 + lq;
        auto read_w = [&](int half, int i, int buf) __attribute__((always_inline)) {
            w[half][i] = __builtin_bit_cast(u32x4_t, pw[buf * BN * 4 + (half * HN + i) * 64]);
        };
        auto read_x = [&](int half, int i, int part, int buf) __attribute__((always_inline)) {
            const u32x4_t v = __builtin_bit_cast(u32x4_t, (part ? px1 : px0)[buf * BM * 8 + (half * HT + i) * 128]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[half][i][part * 4 + e] = (int)v[e];
        };
        auto read_ws = [&](int half, int i, int sbuf) __attribute__((always_inline)) { wsc[half][i] = psw[sbuf * (BM + BN) * 4 + (half * HN + i) * 64]; };
        auto read_xs = [&](int half, int i, int sbuf) __attribute__((always_inline)) { xsc[half][i] = psx[sbuf * (BM + BN) * 4 + (half * HT + i) * 64]; };
        auto pin = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
        constexpr int Q = HN * HT, GL = GX + GW;
        constexpr auto load_slot = [](int j) { return (2 * j + 2) * 2 * Q / (2 * GL + 1); };
        static_assert(load_slot(0) >= 1 && load_slot(GL - 1) < 2 * Q && 2 * Q > GL, "every load behind an MFMA of its own, none behind the first");
        // Quadrant (half wh of W, half xh of X) on byte S of the scales; `beside(i)` is issued behind MFMA i.
        auto quadrant = [&](auto sc, int wh, int xh, auto beside) __attribute__((always_inline)) {
            for_each<0, Q>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = ic.value, nb = i / HT, tb = nb % 2 ? HT - 1 - i % HT : i % HT;
                mma_scaled<sc.value>(acc[wh * HN + nb][xh * HT + tb], w[wh][nb], x[xh][tb], wsc[wh][nb], xsc[xh][tb]);
                pin();
                beside(ic);
                pin();
            });
        };
        auto stage = [&](int kt, int sbuf, auto sc) __attribute__((always_inline)) {
            constexpr int s = sc.value, buf = s % D, next = (s + 1) % D, a = s & 1, b = a ^ 1;
            // first quadrant: the other halves of this stage, X's first
            quadrant(sc, 0, a, [&](auto ic) __attribute__((always_inline)) {
                constexpr int i = ic.value, R = 2 * HT + HN;
                for_each<i * R / Q, (i + 1) * R / Q>([&](auto jc) __attribute__((always_inline)) {
                    constexpr int j = jc.value;
                    if constexpr (j < 2 * HT) {
                        read_x(b, j / 2, j % 2, buf);
                        if constexpr (s == 0 && j % 2 == 0) read_xs(b, j / 2, sbuf);
                    } else {
                        read_w(1, j - 2 * HT, buf);
                        if constexpr (s == 0) read_ws(1, j - 2 * HT, sbuf);
                    }
                });
            });
            next_desc(kt + D);
            quadrant(sc, 0, b, [&](auto) __attribute__((always_inline)) {});
            wait_vm_barrier<(D - 2) * GL>();  // the next stage is there (the D - 2 behind it may not be); this one has been read by every wave
            if (is_tail(kt + 1)) zero_tail(next);
            if constexpr (s == 0) {
                if (kt + 4 < KT) request_scales((kt >> 2) + 1);
            }
            if constexpr (s == 2) {  // (there since this barrier at the latest; read from stage 3's on; that buffer was last read in stage 0)
                if (kt + 2 < KT) order_scales((kt >> 2) + 1);
            }
            // third and fourth quadrant: W0, then Xb of the next stage; stage kt + D is requested
            auto loads = [&](auto ic) __attribute__((always_inline)) {  // (i: of 2 Q MFMAs; where a load goes is set one MFMA ahead)
                constexpr int i = ic.value;
                for_each<0, GL>([&](auto jc) __attribute__((always_inline)) {
                    if constexpr (load_slot(jc.value) == i) load(jc);
                });
                for_each<0, GL>([&](auto jc) __attribute__((always_inline)) {
                    if constexpr (load_slot(jc.value) == i + 1) load_base(jc, buf);
                });
            };
            quadrant(sc, 1, b, [&](auto ic) __attribute__((always_inline)) {
                constexpr int i = ic.value;
                for_each<i * HN / Q, (i + 1) * HN / Q>([&](auto jc) __attribute__((always_inline)) {
                    read_w(0, jc.value, next);
                    if constexpr (s == 3) read_ws(0, jc.value, sbuf ^ 1);
                });
                loads(ic);
            });
            quadrant(sc, 1, a, [&](auto ic) __attribute__((always_inline)) {
                constexpr int i = ic.value;
                for_each<i * 2 * HT / Q, (i + 1) * 2 * HT / Q>([&](auto jc) __attribute__((always_inline)) {
                    read_x(b, jc.value / 2, jc.value % 2, next);
                    if constexpr (s == 3 && jc.value % 2 == 0) read_xs(b, jc.value / 2, sbuf ^ 1);
                });
                loads(std::integral_constant<int, i + Q>{});
            });
        };
        wait_vm_barrier<(D - 1) * GL>();  // the scales and the first stage are there
        order_scales(0);
        __syncthreads();
        if (is_tail(0)) zero_tail(0);
#pragma unroll
        for (int i = 0; i < HN; ++i) read_w(0, i, 0), read_ws(0, i, 0);
#pragma unroll
        for (int i = 0; i < HT; ++i) read_x(0, i, 0, 0), read_x(0, i, 1, 0), read_xs(0, i, 0);
#pragma clang loop unroll(disable)
        for (int kt = 0; kt < KT; kt += 4) {
            for_each<0, 4>([&](auto sc) __attribute__((always_inline)) {
                if (kt + sc.value < KT) stage(kt + sc.value, (kt >> 2) & 1, sc);
            });
        }
    }
    // ---- extension: stage e is in the LDS of stage KT + e -------------------------------------------------------------------
    if (!SPLIT && n_seg > 0) {
        int buf = KT % D;
        while (span[0] != 0) {
            const int lo = span[0] & 0xffff, hi = span[0] >> 16;
            chunk_t w[NBN], x[NBT];
#pragma unroll
            for (int nb = 0; nb < NBN; ++nb) w[nb] = read_here(sW + buf * BN * 4 + w_at(wn0 + lr, lq) + nb * 64);
#pragma unroll
            for (int tb = 0; tb < NBT; ++tb) x[tb] = read_here(sX + buf * BM * 8 + x_at(wm0 + lr, lq) + tb * 128);
#pragma unroll
            for (int tb = 0; tb < NBT; ++tb) {
                const int t0 = wm0 + tb * 16;
                if (lo < t0 + 16 && hi > t0) {
#pragma unroll
                    for (int nb = 0; nb < NBN; ++nb) Elem<E>::mma_step(acc[nb][tb], w[nb], x[tb], 0);
                }
            }
            wait_vm_barrier<(D - 2) * (GX + GW)>();  // the next one is there; this one has been read by every wave
            next_desc(KT);  // (no bytes behind the last one: the counts stay what they are)
            for_each<0, GX + GW>([&](auto jc) __attribute__((always_inline)) { load_base(jc, buf), load_settled(jc); });
            buf = buf + 1 == D ? 0 : buf + 1;
        }
    }
    settle();
    wait_vm<0>();  // (loads past the end: none may arrive in LDS that is another workgroup's by then)

    // ---- the single store of Y (or of a split's partial sums, in fp32) -----------------------------------------------------
    constexpr int NP = NBN / 2;
    const int pc = n0 + wn0 + pair_column(lane);
    if constexpr (SPLIT) {
        float *P = p.P + (int64_t)blockIdx.y * p.T * p.ldp;
#pragma unroll
        for (int tb = 0; tb < NBT; ++tb) {
            const int t = wm0 + tb * 16 + lr;
            float *prow = P + (int64_t)srow[t] * p.ldp;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float v[8];
                pair_columns(acc[2 * i][tb], acc[2 * i + 1][tb], v);
                if (m0 + t < p.T) store_columns(prow, pc + i * 32, g.N, v);
            }
        }
    } else {
        E *Y = static_cast<E *>(g.Y);
        if (g.D == nullptr) {
#pragma unroll
            for (int tb = 0; tb < NBT; ++tb) {
                const int t = wm0 + tb * 16 + lr;
                E *yrow = Y + (int64_t)srow[t] * g.ldy;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    float v[8];
                    pair_columns(acc[2 * i][tb], acc[2 * i + 1][tb], v);
                    if (m0 + t < p.T) store_columns(yrow, pc + i * 32, g.N, v);
                }
            }
        } else {
            // The term is read AHEAD row blocks before the stores that it is added into, and only where a block holds such a row: 8 MB instead of
            // 53 at 1216 rows of which 186 take it, 4096 -> 11008.  The time there is the same, 64.9 us and 64.3 with one block ahead and every
            // block read: it is the chain of reads at the tile's end, 8.5 us over a table that no row uses (56), that costs.
            constexpr int AHEAD = NBT > 4 ? 3 : 2;
            chunk_t term[AHEAD + 1][2 * NP];
            auto fetch = [&](int tb, chunk_t(&d)[2 * NP]) __attribute__((always_inline)) {
                const int t = wm0 + tb * 16 + lr;
                const bool has = use_d[t] != 0;
                if (__builtin_amdgcn_ballot_w64(has) == 0) return;
                const float *drow = g.D + (has ? (int64_t)srow[t] * g.ldd : 0);
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const float *src = drow + min(pc + i * 32, (int)g.ldd - 8);  // (columns past N: loaded, never stored)
                    d[2 * i] = load_chunk(src);
                    d[2 * i + 1] = load_chunk(src + 4);
                }
            };
            auto add4 = [](float *v, bool has, const chunk_t &d) __attribute__((always_inline)) {
                v[0] += has ? __uint_as_float(d.x) : 0.f;
                v[1] += has ? __uint_as_float(d.y) : 0.f;
                v[2] += has ? __uint_as_float(d.z) : 0.f;
                v[3] += has ? __uint_as_float(d.w) : 0.f;
            };
#pragma unroll
            for (int tb = 0; tb < AHEAD; ++tb) fetch(tb, term[tb]);
#pragma unroll
            for (int tb = 0; tb < NBT; ++tb) {
                const int t = wm0 + tb * 16 + lr;
                const bool ok = m0 + t < p.T, has = use_d[t] != 0;
                E *yrow = Y + (int64_t)srow[t] * g.ldy;
                if (tb + AHEAD < NBT) fetch(tb + AHEAD, term[(tb + AHEAD) % (AHEAD + 1)]);
                const chunk_t(&d)[2 * NP] = term[tb % (AHEAD + 1)];
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    float v[8];
                    pair_columns(acc[2 * i][tb], acc[2 * i + 1][tb], v);
                    add4(v, has, d[2 * i]);
                    add4(v + 4, has, d[2 * i + 1]);
                    if (ok) store_columns(yrow, pc + i * 32, g.N, v);
                }
            }
        }
    }
}

// Workgroup -> tile: consecutive ids go round the 8 XCDs, each walks a contiguous range in groups of group_m row tiles.
__device__ __forceinline__ bool tile_of(int id, int tiles_m, int tiles_n, int group_m, int *pm, int *pn) {
    const int total = tiles_m * tiles_n;
    const int per_xcd = (total + 7) >> 3;
    const int lin = (id & 7) * per_xcd + (id >> 3);
    if (lin >= total) return false;
    const int width = group_m * tiles_n;
    const int first_m = lin / width * group_m;
    const int gsz = min(tiles_m - first_m, group_m);
    *pm = first_m + (lin % width) % gsz;
    *pn = (lin % width) / gsz;
    return true;
}

template <int BM, int BN, int PARTS, bool SPLIT>
__global__ __launch_bounds__(256) void mx_gemm_kernel(MxGemmArgs p, int tiles_m, int tiles_n, int group_m) {
    int pm, pn;
    if (tile_of(blockIdx.x, tiles_m, tiles_n, group_m, &pm, &pn)) mx_gemm_tile<BM, BN, PARTS, SPLIT>(p, pm * BM, pn);
}

// 256 x 256 tiles, and behind them tiles of 128 x 256 for the last, at most 128 rows: the chip's last round is then that much shorter, or
// there is none (7500 rows 4096 -> 11008: 1247 tiles and 43 of half the work in five rounds, where 1290 take a sixth for ten of them).
template <int PARTS>
__global__ __launch_bounds__(256) void mx_gemm_kernel_mixed(MxGemmArgs p, int tiles_m, int tiles_n, int group_m, int first_small) {
    int pm, pn;
    if ((int)blockIdx.x >= first_small)
        mx_gemm_tile<128, 256, PARTS, false>(p, tiles_m * 256, (int)blockIdx.x - first_small);
    else if (tile_of(blockIdx.x, tiles_m, tiles_n, group_m, &pm, &pn))
        mx_gemm_tile<256, 256, PARTS, false>(p, pm * 256, pn);
}

template <int BM, int BN, int PARTS, bool SPLIT>
hipError_t launch_s(const MxGemmArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    MxGemmArgs a = a0;
    const int tiles_m = (a.T + BM - 1) / BM;
    int tiles_n = 0;
    for (int i = 0; i < a.n_sets; ++i) {
        a.set[i].tile0 = tiles_n;
        tiles_n += (a.set[i].N + BN - 1) / BN;
    }
    const long total = (long)tiles_m * tiles_n;
    if (total <= 0) return hipSuccess;
    return launch_kernel(mx_gemm_kernel<BM, BN, PARTS, SPLIT>, dim3((unsigned)((total + 7) / 8 * 8), SPLIT ? (unsigned)a.split_k : 1u), dim3(256),
                         MxTile<BM, BN>::smem, stream, timer, a, tiles_m, tiles_n, 8);
}
template <int BM, int BN, int PARTS>
hipError_t launch_p(const MxGemmArgs &a, hipStream_t stream, const KernelTimer *timer) {
    return a.split_k > 1 ? launch_s<BM, BN, PARTS, true>(a, stream, timer) : launch_s<BM, BN, PARTS, false>(a, stream, timer);
}
template <int BM, int BN>
hipError_t launch_t(const MxGemmArgs &a, hipStream_t stream, const KernelTimer *timer) {
    return a.parts == 2 ? launch_p<BM, BN, 2>(a, stream, timer) : launch_p<BM, BN, 1>(a, stream, timer);
}
template <int BM, int BN>
hipError_t init_t() {
    const void *const kernels[4] = {reinterpret_cast<const void *>(mx_gemm_kernel<BM, BN, 1, false>), reinterpret_cast<const void *>(mx_gemm_kernel<BM, BN, 1, true>),
                                    reinterpret_cast<const void *>(mx_gemm_kernel<BM, BN, 2, false>), reinterpret_cast<const void *>(mx_gemm_kernel<BM, BN, 2, true>)};
    for (const void *k : kernels) {
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)MxTile<BM, BN>::smem);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr size_t kMixedSmem = MxTile<128, 256>::smem > MxTile<256, 256>::smem ? MxTile<128, 256>::smem : MxTile<256, 256>::smem;
template <int PARTS>
hipError_t launch_mixed(const MxGemmArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    MxGemmArgs a = a0;
    const int tiles_m = a.T / 256, rest = a.T % 256;
    if (tiles_m < 1 || rest < 1 || rest > 128 || a.split_k > 1) return hipErrorInvalidValue;
    int tiles_n = 0;
    for (int i = 0; i < a.n_sets; ++i) {
        a.set[i].tile0 = tiles_n;
        tiles_n += (a.set[i].N + 255) / 256;
    }
    const long big = ((long)tiles_m * tiles_n + 7) / 8 * 8;
    return launch_kernel(mx_gemm_kernel_mixed<PARTS>, dim3((unsigned)(big + tiles_n)), dim3(256), kMixedSmem, stream, timer, a, tiles_m, tiles_n, 8, (int)big);
}
hipError_t init_mixed() {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(mx_gemm_kernel_mixed<1>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMixedSmem);
    if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void *>(mx_gemm_kernel_mixed<2>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMixedSmem);
    return e;
}

}  // namespace

hipError_t init_mx_gemm_kernels() {
    hipError_t e = init_t<256, 256>();
    if (e == hipSuccess) e = init_t<128, 256>();
    if (e == hipSuccess) e = init_t<128, 128>();
    if (e == hipSuccess) e = init_mixed();
    return e;
}

hipError_t launch_mx_gemm(const MxGemmArgs &a, int variant, hipStream_t stream, const KernelTimer *timer) {
    if (!(a.T > 0 && a.K > 0 && a.K % kMxBlock == 0 && a.n_sets >= 1 && a.n_sets <= kMaxGemmSets && a.Xq && a.Xs && (a.parts == 1 || a.parts == 2)))
        return hipErrorInvalidValue;
    const int blocks = a.K / kMxBlock;
    if (a.parts == 2 && (a.part_bytes < a.K || a.part_scales < blocks)) return hipErrorInvalidValue;
    if (a.split_k > 1) {
        if (a.n_sets != 1 || a.set[0].B || a.set[0].D || !a.P || a.ldp < a.set[0].N || (a.ldp & 7) || a.chunk_blocks <= 0 || a.chunk_blocks % 16 ||
            (long)a.chunk_blocks * (a.split_k - 1) >= blocks || (long)a.chunk_blocks * a.split_k < blocks)
            return hipErrorInvalidValue;
    }
    switch (variant) {
        case kMxTile256x256:
            return launch_t<256, 256>(a, stream, timer);
        case kMxTile128x256:
            return launch_t<128, 256>(a, stream, timer);
        case kMxTile128x128:
            return launch_t<128, 128>(a, stream, timer);
        case kMxTileMixed:
            return a.parts == 2 ? launch_mixed<2>(a, stream, timer) : launch_mixed<1>(a, stream, timer);
        default:
            return hipErrorInvalidValue;
    }
}

}  // namespace lora
