// Decode-sized batches (T <= 128 rows) on a 4-bit backbone: the first of the decode path's two launches, which streams W
// and the used A_a against X, slice by slice of the contraction axis, and leaves fp32 partial tiles; the second (reduction or
// finishing kernel, decode_kernels.hip) is the decode path's own and reads the same tiles.
//
//     P[n, t] = sum over a slice of  e2m1(W[n, k]) 2^(s[n, k/32] - 127)  X[t, k]
//
// Bound by the stream of W -- half a byte a value and a byte for 32 of them -- by the partial tiles, and, the fewer rows there are, by the
// chain of one wave's instructions; so the weights are never taken apart by arithmetic.  Activations in bf16: the hardware's
// conversion turns two 4-bit values and their scale into two bf16 values, exactly, and the products run on 16x16x32 bf16
// MFMAs.  Activations in 8 bits: block-scaled 16x16x128 MFMAs take both as they are (operand layout: mx_gemm_kernels.hip).
//
// A wave has 16 rows of W and a slice of SC chunks of 8 values: it requests all its weights at once, 8 rows x 128 bytes
// an instruction, and turns them into operand layout through a wave-private, XOR-swizzled LDS buffer, as the decode path
// does for bf16.  A lane's 16 bytes there are one whole block -- row lane % 16, block 4 q + lane / 16 -- so it needs one scale; in
// bf16 they feed four MFMAs, the j-th of which takes values 8 j .. 8 j + 7 of four blocks, from both sides.
//
// The rows of the used A_a (bf16, slices of 512 values, X in bf16) are workgroups of their own in front of the others: their X is another
// where the backbone's comes in 8 bits.
#include <type_traits>

#include "mx_common.hiph"

namespace lora {
namespace {

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A pair of bf16 values (as bits) of byte `B` / half `B` of a dword of codes.
template <int B>
__device__ __forceinline__ unsigned open_fp4(unsigned codes, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
__device__ __forceinline__ chunk_t open_fp4x8(unsigned codes, float scale) {
    return make_uint4(open_fp4<0>(codes, scale), open_fp4<1>(codes, scale), open_fp4<2>(codes, scale), open_fp4<3>(codes, scale));
}
template <typename F>
__device__ __forceinline__ void for_pair(F &&f) {
    f(std::integral_constant<int, 0>{});
    f(std::integral_constant<int, 1>{});
}

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kExtChunks = 64;  // chunks of X per slice of the extension rows

// X in bf16, a slice of SC chunks: requested, and put into LDS, chunk c of row t at t * SC + (c ^ mx_row_swizzle(t)) (zeros past T and K).
template <int TBLK, int SC, int MINT>
struct XSlice {
    static constexpr int IT = (TBLK * 16 * SC + MINT - 1) / MINT;  // (with the fewest threads of a workgroup)
    chunk_t v[IT];
    __device__ __forceinline__ void request(const DecodeArgs &p, int kc0, int kchunks) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int idx = (int)threadIdx.x + it * (int)blockDim.x;
            const int row = min(idx / SC, p.T - 1), c = min(kc0 + idx % SC, kchunks - 1);
            v[it] = load_chunk(static_cast<const __bf16 *>(p.X) + (int64_t)row * p.ldx + c * 8);
        }
    }
    __device__ __forceinline__ void stage(chunk_t *xs, const DecodeArgs &p, int kc0, int kchunks) const {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int idx = (int)threadIdx.x + it * (int)blockDim.x;
            const int row = idx / SC, c = idx % SC;
            if (idx < TBLK * 16 * SC) xs[row * SC + (c ^ mx_row_swizzle(row))] = keep_if(row < p.T && kc0 + c < kchunks, v[it]);
        }
    }
};

// TBLK: 16-row blocks of the batch.  SC: chunks of 8 values per slice of the backbone.  X8: its activations come in 8 bits.
template <int TBLK, int SC, bool X8>
__global__ __launch_bounds__(kDecodeMaxWaves * 64) void mx_decode_stream_kernel(MxDecodeArgs a) {
    typedef __bf16 E;
    constexpr int XROWS = TBLK * 16;
    constexpr int NST = SC / 32;  // stages of 128 bytes of a weight row
    constexpr int MINT = mx_fewest_waves(TBLK, SC) * 64;
    constexpr bool MASKED = TBLK < 8;

    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const DecodeArgs &p = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nthreads = blockDim.x, nw = nthreads >> 6;
    const int li = lane & 15, lg = lane >> 4;
    const int status = p.plan.scalars[kScStatus];
    const int kchunks = p.K / 8;
    const int wr = lane >> 3, wc = lane & 7;  // load slot: row wr + 8 i of the block, chunk wc of a 128-byte stage
    chunk_t *buf = reinterpret_cast<chunk_t *>(smem) + wave * 128;
    chunk_t *xs = reinterpret_cast<chunk_t *>(smem) + nw * 128;
    int wdst[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = wr + 8 * i;
        wdst[i] = row * 8 + (wc ^ ((row >> 1) & 7));
    }
    const int rsrc = li * 8, rswz = (li >> 1) & 7, lsw = mx_row_swizzle(li);
    f32x4_t acc[TBLK];
#pragma unroll
    for (int tb = 0; tb < TBLK; ++tb) acc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    float4 *P4;
    unsigned keep;  // token blocks whose results this lane stores, one bit each
    if ((int)blockIdx.x < a.ext_wgs) {
        const int slice = blockIdx.x % p.ks_ext;
        int grp = blockIdx.x / p.ks_ext;
        const int si = grp / a.ext_groups;
        grp -= si * a.ext_groups;
        const DecodeSet &set = p.set[si];
        const int kc0 = slice * kExtChunks;
        const int blk = grp * nw + wave;
        const int nrec = p.plan.scalars[kScExtTotal] >> 3;  // records of 8 ranks
        const bool valid = set.A != nullptr && blk < p.nbe && blk * 2 < nrec;
        int4 rec[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};
        if (valid) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (blk * 2 + i < nrec) rec[i] = reinterpret_cast<const int4 *>(p.plan.ext_rec)[blk * 2 + i];
        }
        int row_ad[TBLK];
#pragma unroll
        for (int tb = 0; tb < TBLK; ++tb) {
            row_ad[tb] = -2;
            if (MASKED && tb * 16 + li < p.T) row_ad[tb] = p.plan.row_adapter[tb * 16 + li];
        }
        XSlice<TBLK, kExtChunks, MINT> xv;
        xv.request(p, kc0, kchunks);
        const char *rowp[2];
        bool rowok[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int ad = rec[i].x, j = rec[i].y & 0xffff;
            const void *ap = ad >= 0 ? set.A[ad] : nullptr;
            if (ad >= 0 && ap == nullptr) atomicMin(&p.plan.scalars[kScEvicted], kErrNotResident);  // slot emptied after the plan
            rowok[i] = ap != nullptr;
            rowp[i] = rowok[i] ? static_cast<const char *>(ap) + (int64_t)(j + wr) * p.K * 2 : static_cast<const char *>(p.X);
        }
        keep = 0;
        if (MASKED) {
            const int own = lg < 2 ? rec[0].x : rec[1].x;
#pragma unroll
            for (int tb = 0; tb < TBLK; ++tb) keep |= row_ad[tb] == own ? 1u << tb : 0u;
        } else {
            keep = (TBLK - 1) * 16 + li < p.T ? (1u << TBLK) - 1u : (1u << (TBLK - 1)) - 1u;
        }
        // (half of the block's 16 KB before X goes to LDS, whose registers the rest takes)
        chunk_t wq[8][2];
        auto load_w = [&](int s) __attribute__((always_inline)) {
            const unsigned off = (unsigned)min(kc0 + s * 8 + wc, kchunks - 1) * 16u;
#pragma unroll
            for (int i = 0; i < 2; ++i) wq[s][i] = load_chunk(rowp[i] + (rowok[i] ? off : 0u));
        };
#pragma unroll
        for (int s = 0; s < 4; ++s) load_w(s);
        xv.stage(xs, p, kc0, kchunks);
        lds_barrier();
        if (!valid || status != 0) return;
        load_w(4);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s + 5 < 8) load_w(s + 5);
            if (kc0 + s * 8 < kchunks) {  // a stage: 8 chunks, 64 values of A_a
                buf[wdst[0]] = keep_if(rowok[0], wq[s][0]);
                buf[wdst[1]] = keep_if(rowok[1], wq[s][1]);
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const chunk_t w = buf[rsrc + ((h * 4 + lg) ^ rswz)];
#pragma unroll
                    for (int tb = 0; tb < TBLK; ++tb)
                        Elem<E>::mma16(acc[tb], w, xs[(tb * 16 + li) * kExtChunks + ((s * 8 + h * 4 + lg) ^ lsw)]);
                }
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            }
        }
        P4 = reinterpret_cast<float4 *>(set.P) + ((int64_t)(blk * p.ks_ext + slice) * TBLK) * 64;
    } else {
        const int wg = (int)blockIdx.x - a.ext_wgs, slice = wg % p.ks;
        int grp = wg / p.ks;
        int si = 0;
        while (si + 1 < a.n && grp >= a.w[si + 1].group0) ++si;
        grp -= a.w[si].group0;
        const DecodeSet &set = p.set[si];
        const MxDecodeSet &w4 = a.w[si];
        const int kc0 = slice * SC;
        const int blk = grp * nw + wave;
        const bool valid = blk < set.nbw;
        const int nblocks = p.K / kMxBlock, kb0 = kc0 / 4;  // blocks of a row; the slice's first
        keep = (TBLK - 1) * 16 + li < p.T ? (1u << TBLK) - 1u : (1u << (TBLK - 1)) - 1u;
        // ---- X first (all of it before any weights: see decode_stream_kernel) ----
        constexpr int PC = SC / 2, SS = SC / 64;  // of X in 8 bits: 16-byte pieces and groups of 16 blocks per slice and row
        constexpr int X8IT = (XROWS * PC + MINT - 1) / MINT, XSIT = (XROWS * SS + MINT - 1) / MINT;
        chunk_t x8v[X8 ? X8IT : 1], x8s[X8 ? XSIT : 1];
        XSlice<X8 ? 1 : TBLK, X8 ? 32 : SC, MINT> xv;
        if constexpr (X8) {
#pragma unroll
            for (int it = 0; it < XSIT; ++it) {
                const int idx = tid + it * nthreads, row = min(idx / SS, p.T - 1);
                x8s[it] = zero_chunk();
                if (idx < XROWS * SS) x8s[it] = mx_load_scales(a.Xs + (int64_t)row * a.ldxs, slice * SS + idx % SS, nblocks);
            }
#pragma unroll
            for (int it = 0; it < X8IT; ++it) {
                const int idx = tid + it * nthreads;
                const int row = min(idx / PC, p.T - 1), c = min(kc0 / 2 + idx % PC, kchunks / 2 - 1);
                x8v[it] = load_chunk(a.Xq + (int64_t)row * a.ldxq + c * 16);
            }
        } else {
            xv.request(p, kc0, kchunks);
        }
        __builtin_amdgcn_s_barrier();
        // ---- all of the wave's weights: 16 rows (those past N are clamped: never read back) ----
        const unsigned char *rowp[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) rowp[i] = w4.Wq + (int64_t)min(blk * 16 + wr + 8 * i, set.N - 1) * w4.ldwq;
        const unsigned char *srow = w4.Ws + (int64_t)min(blk * 16 + li, set.N - 1) * w4.ldws;
        chunk_t wq[NST][2];
        unsigned sq[NST * 2];  // scales: four blocks of the lane's row each
#pragma unroll
        for (int s = 0; s < NST; ++s) {
            const unsigned off = (unsigned)min(kb0 + s * 8 + wc, nblocks - 1) * 16u;
#pragma unroll
            for (int i = 0; i < 2; ++i) wq[s][i] = load_chunk(rowp[i] + off);
#pragma unroll
            for (int q = 0; q < 2; ++q) sq[s * 2 + q] = mx_load_u32(srow + (min(kb0 + s * 8 + q * 4, nblocks - 1) & ~3));
        }
        // X in 8 bits in LDS: piece c of row t at t * PC + (c ^ (t & 15)); behind it the scales, in the order of the lanes (mx_transpose_scales)
        unsigned *xsc = reinterpret_cast<unsigned *>(xs + XROWS * PC);
        if constexpr (X8) {
#pragma unroll
            for (int it = 0; it < XSIT; ++it) {
                const int idx = tid + it * nthreads;
                if (idx < XROWS * SS) reinterpret_cast<chunk_t *>(xsc)[idx] = mx_transpose_scales(x8s[it]);
            }
#pragma unroll
            for (int it = 0; it < X8IT; ++it) {
                const int idx = tid + it * nthreads;
                const int row = idx / PC, c = idx % PC;
                if (idx < XROWS * PC) xs[row * PC + (c ^ (row & 15))] = keep_if(row < p.T && kc0 / 2 + c < kchunks / 2, x8v[it]);
            }
        } else {
            xv.stage(xs, p, kc0, kchunks);
        }
        lds_barrier();  // (LDS traffic only: the weight loads stay in flight across it)
        if (!valid || status != 0) return;
        unsigned xscale[TBLK];
#pragma unroll
        for (int s = 0; s < NST; ++s) {
            if (kb0 + s * 8 >= nblocks) break;
            buf[wdst[0]] = wq[s][0];
            buf[wdst[1]] = wq[s][1];
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            if constexpr (X8) {
                if (s % 2 == 0) {
#pragma unroll
                    for (int tb = 0; tb < TBLK; ++tb) xscale[tb] = xsc[((tb * 16 + li) * SS + s / 2) * 4 + lg];
                }
            }
            for_pair([&](auto qc) __attribute__((always_inline)) {
                constexpr int q = qc.value;
                const chunk_t w = buf[rsrc + ((q * 4 + lg) ^ rswz)];
                // (past K the codes are some of this row's, the scale 2^-127: finite, and X holds zeros there)
                const unsigned sb = kb0 + s * 8 + q * 4 + lg < nblocks ? (sq[s * 2 + q] >> (8 * lg)) & 255u : 0u;
                if constexpr (X8) {
                    const i32x8_t wo{(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
#pragma unroll
                    for (int tb = 0; tb < TBLK; ++tb) {
                        const chunk_t *xr = xs + (tb * 16 + li) * PC;
                        const chunk_t u = xr[(s * 16 + q * 8 + lg) ^ li], v = xr[(s * 16 + q * 8 + 4 + lg) ^ li];
                        const i32x8_t xo{(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
                        if (s % 2 == 0)
                            acc[tb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wo, xo, acc[tb], 4, 0, 0, (int)sb, q, (int)xscale[tb]);
                        else
                            acc[tb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wo, xo, acc[tb], 4, 0, 0, (int)sb, q + 2, (int)xscale[tb]);
                    }
                } else {
                    const float sc = __uint_as_float(sb << 23);
                    const unsigned wd[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const chunk_t op = open_fp4x8(wd[j], sc);
#pragma unroll
                        for (int tb = 0; tb < TBLK; ++tb)
                            Elem<E>::mma16(acc[tb], op, xs[(tb * 16 + li) * SC + ((s * 32 + q * 16 + lg * 4 + j) ^ lsw)]);
                    }
                }
            });
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        }
        P4 = reinterpret_cast<float4 *>(set.P) + (((int64_t)p.nbe_cap * p.ks_ext + (int64_t)blk * p.ks + slice) * TBLK) * 64;
    }
    // acc[tb][e] = D[weight row of the block lg * 4 + e][token tb * 16 + li]: token-major KiB tiles, as decode_stream_kernel's
    P4 += li * 4 + lg;
#pragma unroll
    for (int tb = 0; tb < TBLK; ++tb)
        if (keep >> tb & 1u) P4[tb * 64] = make_float4(acc[tb][0], acc[tb][1], acc[tb][2], acc[tb][3]);
}

// Bytes of LDS: the waves' buffers, and X of either kind of workgroup (its scales take 1/32 of what it does in 8 bits).
template <int TBLK, int SC, bool X8>
constexpr size_t mx_stream_smem(int waves) {
    const size_t ext = (size_t)TBLK * 16 * kExtChunks * 16, base = X8 ? (size_t)TBLK * 16 * SC * 8 + (size_t)TBLK * 16 * (SC / 64) * 16 : (size_t)TBLK * 16 * SC * 16;
    return (size_t)waves * 2048 + (ext > base ? ext : base);
}
template <int TBLK, int SC, bool X8>
constexpr bool kFits = TBLK * 16 * SC * (X8 ? 8 : 16) <= 128 * 1024 && SC <= kMxMostChunks;

template <int TBLK, int SC, bool X8>
hipError_t launch_t(const MxDecodeArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    if constexpr (kFits<TBLK, SC, X8>) {
        MxDecodeArgs a = a0;
        const int w = a.d.waves;
        if (w < mx_fewest_waves(TBLK, SC) || w > kDecodeMaxWaves) return hipErrorInvalidValue;
        a.ext_groups = (a.d.nbe + w - 1) / w;
        a.ext_wgs = a.n * a.ext_groups * a.d.ks_ext;
        long groups = 0;
        for (int i = 0; i < a.n; ++i) {
            a.w[i].group0 = (int32_t)groups;
            groups += (a.d.set[i].nbw + w - 1) / w;
        }
        const long grid = a.ext_wgs + groups * a.d.ks;
        return launch_kernel(mx_decode_stream_kernel<TBLK, SC, X8>, dim3((unsigned)grid), dim3(w * 64), mx_stream_smem<TBLK, SC, X8>(w), stream, timer, a);
    } else {
        return hipErrorInvalidValue;
    }
}
template <int TBLK, int SC, bool X8>
hipError_t init_t() {
    if constexpr (kFits<TBLK, SC, X8>)
        return hipFuncSetAttribute(reinterpret_cast<const void *>(mx_decode_stream_kernel<TBLK, SC, X8>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)mx_stream_smem<TBLK, SC, X8>(kDecodeMaxWaves));
    return hipSuccess;
}
template <int TBLK, bool X8>
hipError_t launch_x(const MxDecodeArgs &a, hipStream_t stream, const KernelTimer *timer) {
    switch (a.d.slice_chunks) {
        case 64:
            return launch_t<TBLK, 64, X8>(a, stream, timer);
        case 128:
            return launch_t<TBLK, 128, X8>(a, stream, timer);
        default:
            return hipErrorInvalidValue;
    }
}
template <int TBLK>
hipError_t launch_b(const MxDecodeArgs &a, hipStream_t stream, const KernelTimer *timer) {
    return a.Xq ? launch_x<TBLK, true>(a, stream, timer) : launch_x<TBLK, false>(a, stream, timer);
}
template <int TBLK>
hipError_t init_b() {
    hipError_t e = init_t<TBLK, 64, false>();
    if (e == hipSuccess) e = init_t<TBLK, 128, false>();
    if (e == hipSuccess) e = init_t<TBLK, 64, true>();
    if (e == hipSuccess) e = init_t<TBLK, 128, true>();
    return e;
}

}  // namespace

hipError_t init_mx_decode_kernels() {
    hipError_t e = init_b<1>();
    if (e == hipSuccess) e = init_b<2>();
    if (e == hipSuccess) e = init_b<3>();
    if (e == hipSuccess) e = init_b<4>();
    if (e == hipSuccess) e = init_b<5>();
    if (e == hipSuccess) e = init_b<6>();
    if (e == hipSuccess) e = init_b<7>();
    if (e == hipSuccess) e = init_b<8>();
    return e;
}

hipError_t launch_mx_decode_stream(const MxDecodeArgs &a, int tblk, hipStream_t stream, const KernelTimer *timer) {
    const DecodeArgs &d = a.d;
    if (!(d.T > (tblk - 1) * 16 && d.T <= tblk * 16 && d.K > 0 && d.K % kMxBlock == 0 && d.nbe >= 0 && d.nbe <= d.nbe_cap && a.n >= 1 &&
          a.n <= kMaxGemmSets && d.slice_chunks > 0 && d.ks == (d.K / 8 + d.slice_chunks - 1) / d.slice_chunks &&
          d.ks_ext == (d.K / 8 + kExtChunks - 1) / kExtChunks && (d.X != nullptr || (a.Xq != nullptr && d.nbe == 0))))
        return hipErrorInvalidValue;
    for (int i = 0; i < a.n; ++i)
        if (!(d.set[i].N > 0 && d.set[i].nbw == (d.set[i].N + 15) / 16 && d.set[i].P != nullptr && a.w[i].Wq != nullptr && a.w[i].Ws != nullptr))
            return hipErrorInvalidValue;
    switch (tblk) {
        case 1:
            return launch_b<1>(a, stream, timer);
        case 2:
            return launch_b<2>(a, stream, timer);
        case 3:
            return launch_b<3>(a, stream, timer);
        case 4:
            return launch_b<4>(a, stream, timer);
        case 5:
            return launch_b<5>(a, stream, timer);
        case 6:
            return launch_b<6>(a, stream, timer);
        case 7:
            return launch_b<7>(a, stream, timer);
        case 8:
            return launch_b<8>(a, stream, timer);
        default:
            return hipErrorInvalidValue;
    }
}

}  // namespace lora
