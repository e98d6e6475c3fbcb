// Decode-sized batches (T <= 128 rows) on a 4-bit backbone: the first of the decode path's two launches, which streams W
// and the used A_a against X, slice by slice of the contraction axis, and leaves fp32 partial tiles; the second (reduction or
// finishing kernel, decode_kernels.hip) is the decode path's own and reads the same tiles.
//
//     P[n, t] = sum over a slice of  e2m1(W[n, k]) 2^(s[n, k/32] - 127)  X[t, k]
//
// Bound by the stream of W -- half a byte a value and a byte for 32 of them -- and, the fewer rows there are, by the chain of one
// wave's instructions; so the weights are never taken apart by arithmetic: the hardware's conversion turns two 4-bit values and
// their scale into two bf16 values, exactly, and the products run on 16x16x32 bf16 MFMAs.  (X in 8 bits is opened the same way,
// exactly, when it is staged in LDS: T x K values against N x K.)
//
// A wave has 16 rows of W and a slice of SC 16-byte chunks of X (8 values each): it requests all its weights at once, 8 rows x
// 128 bytes an instruction, and turns them into operand layout through a wave-private, XOR-swizzled LDS buffer, as the
// decode path does for bf16.  A lane's 16 bytes there are one whole block -- row lane % 16, block 4 q + lane / 16 -- so it
// needs one scale, and feeds four MFMAs: the j-th takes values 8 j .. 8 j + 7 of four blocks, from both sides.
// Slices of 1024 instead of 512 values halve the partial tiles (4 bytes x T x N a slice, written and read; the weights of a slice
// of 512 are 256 N bytes); they are taken where that still leaves a workgroup for every CU (see launch rule in mx_api.hiph).
#include "mx_kernels.h"

namespace lora {
namespace {

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned load_u32(const void *p) { return *(const __attribute__((address_space(1))) unsigned *)p; }

// A pair of bf16 values (as bits) of byte `B` / half `B` of a dword of codes.
template <int B>
__device__ __forceinline__ unsigned open_fp4(unsigned codes, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
__device__ __forceinline__ chunk_t open_fp4x8(unsigned codes, float scale) {
    return make_uint4(open_fp4<0>(codes, scale), open_fp4<1>(codes, scale), open_fp4<2>(codes, scale), open_fp4<3>(codes, scale));
}
__device__ __forceinline__ chunk_t open_fp8x8(unsigned lo, unsigned hi, float scale) {
    return make_uint4(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)));
}

// TBLK: 16-row blocks of the batch.  SC: chunks of X per slice (64 or 128).  X8: the base product's activations come in 8 bits.
template <int TBLK, int SC, bool X8>
__global__ __launch_bounds__(kDecodeMaxWaves * 64) void mx_decode_stream_kernel(MxDecodeArgs a) {
    typedef __bf16 E;
    constexpr int XROWS = TBLK * 16;
    constexpr int MINT = kDecodeMinWaves * 64;           // fewest threads of a workgroup
    constexpr int XIT = XROWS * SC / MINT;               // chunk loads per thread that cover the X slice in bf16
    constexpr int X8IT = (XROWS * SC / 2 + MINT - 1) / MINT;  // 16-byte loads that cover it in 8 bits
    constexpr int NST = SC / 32;                         // stages of 128 bytes of a weight row
    constexpr bool MASKED = TBLK < 8;

    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    chunk_t *xs = reinterpret_cast<chunk_t *>(smem);  // [XROWS][SC], chunk c of row t at t * SC + (c ^ (t & 15))
    chunk_t *wstage = xs + XROWS * SC;                // [waves][128]

    const DecodeArgs &p = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nthreads = blockDim.x, nw = nthreads >> 6;
    const int li = lane & 15, lg = lane >> 4;
    const int slice = blockIdx.x % p.ks;
    int grp = blockIdx.x / p.ks;
    int si = 0;
    while (si + 1 < a.n && grp >= a.w[si + 1].group0) ++si;
    grp -= a.w[si].group0;
    const DecodeSet &set = p.set[si];
    // Workgroups of extension rows (rows of the used A_a) come first: their X is in bf16 whatever the others' is.
    const bool is_ext = grp < a.ext_groups;
    const int status = p.plan.scalars[kScStatus];

    const int kchunks = p.K / 8;
    const int kc0 = slice * SC;
    const int wr = lane >> 3, wc = lane & 7;  // load slot: row wr + 8 i of the block, chunk wc of a 128-byte stage
    chunk_t *buf = wstage + wave * 128;
    int wdst[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = wr + 8 * i;
        wdst[i] = row * 8 + (wc ^ ((row >> 1) & 7));
    }
    const int rsrc = li * 8, rswz = (li >> 1) & 7;
    f32x4_t acc[TBLK];
#pragma unroll
    for (int tb = 0; tb < TBLK; ++tb) acc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // X slice in bf16: request, and put into LDS (zeros past T and K)
    chunk_t xv[X8 ? (XIT > X8IT ? XIT : X8IT) : XIT];
    auto request_x = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int it = 0; it < XIT; ++it) {
            const int idx = tid + it * nthreads;
            const int row = min(idx / SC, p.T - 1), c = min(kc0 + idx % SC, kchunks - 1);
            xv[it] = load_chunk(static_cast<const E *>(p.X) + (int64_t)row * p.ldx + c * 8);
        }
    };
    auto stage_x = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int it = 0; it < XIT; ++it) {
            const int idx = tid + it * nthreads;
            const int row = idx / SC, c = idx % SC;
            if (idx < XROWS * SC) xs[row * SC + (c ^ (row & 15))] = keep_if(row < p.T && kc0 + c < kchunks, xv[it]);
        }
    };

    int pblk;
    unsigned keep;  // token blocks whose results this lane stores, one bit each
    if (is_ext) {
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
        request_x();
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
        stage_x();
        lds_barrier();
        if (!valid || status != 0) return;
        pblk = blk;
        const int nstages = (min(SC, kchunks - kc0) + 7) >> 3;  // of 8 chunks: 64 values of A_a
        for (int s0 = 0; s0 < nstages; s0 += 8) {
            chunk_t wq[8][2];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const unsigned off = (unsigned)min(kc0 + (s0 + s) * 8 + wc, kchunks - 1) * 16u;
#pragma unroll
                for (int i = 0; i < 2; ++i) wq[s][i] = load_chunk(rowp[i] + (rowok[i] ? off : 0u));
            }
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                if (s0 + s < nstages) {
                    buf[wdst[0]] = keep_if(rowok[0], wq[s][0]);
                    buf[wdst[1]] = keep_if(rowok[1], wq[s][1]);
                    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const chunk_t w = buf[rsrc + ((h * 4 + lg) ^ rswz)];
#pragma unroll
                        for (int tb = 0; tb < TBLK; ++tb)
                            Elem<E>::mma16(acc[tb], w, xs[(tb * 16 + li) * SC + (((s0 + s) * 8 + h * 4 + lg) ^ li)]);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
                }
            }
        }
    } else {
        const int blk = (grp - a.ext_groups) * nw + wave;
        const bool valid = blk < set.nbw;
        const MxDecodeSet &w4 = a.w[si];
        const int nblocks = p.K / kMxBlock, kb0 = kc0 / 4;  // blocks of a row; the slice's first
        // ---- X first (all of it before any weights: see decode_stream_kernel) ----
        unsigned xsc[X8 ? X8IT : 1];
        if constexpr (X8) {
#pragma unroll
            for (int it = 0; it < X8IT; ++it) {
                const int idx = tid + it * nthreads;
                const int row = min(idx / (SC / 2), p.T - 1), c = min(kc0 / 2 + idx % (SC / 2), kchunks / 2 - 1);
                xv[it] = load_chunk(a.Xq + (int64_t)row * a.ldxq + c * 16);
                xsc[it] = a.Xs[(int64_t)row * a.ldxs + (c >> 1)];
            }
        } else {
            request_x();
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
            for (int q = 0; q < 2; ++q) sq[s * 2 + q] = load_u32(srow + (min(kb0 + s * 8 + q * 4, nblocks - 1) & ~3));
        }
        keep = (TBLK - 1) * 16 + li < p.T ? (1u << TBLK) - 1u : (1u << (TBLK - 1)) - 1u;
        if constexpr (X8) {
#pragma unroll
            for (int it = 0; it < X8IT; ++it) {
                const int idx = tid + it * nthreads;
                const int row = idx / (SC / 2), c = idx % (SC / 2) * 2;  // two chunks
                if (idx < XROWS * (SC / 2)) {
                    const bool ok = row < p.T && kc0 + c < kchunks;
                    const float sc = __uint_as_float(xsc[it] << 23);
                    xs[row * SC + (c ^ (row & 15))] = keep_if(ok, open_fp8x8(xv[it].x, xv[it].y, sc));
                    xs[row * SC + ((c + 1) ^ (row & 15))] = keep_if(ok, open_fp8x8(xv[it].z, xv[it].w, sc));
                }
            }
        } else {
            stage_x();
        }
        lds_barrier();  // (LDS traffic only: the weight loads stay in flight across it)
        if (!valid || status != 0) return;
        pblk = blk + p.nbe_cap;
#pragma unroll
        for (int s = 0; s < NST; ++s) {
            if (kb0 + s * 8 >= nblocks) break;
            buf[wdst[0]] = wq[s][0];
            buf[wdst[1]] = wq[s][1];
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const chunk_t w = buf[rsrc + ((q * 4 + lg) ^ rswz)];
                // (past K the codes are some of this row's, the scale 2^-127: finite, and X holds zeros there)
                const unsigned sb = kb0 + s * 8 + q * 4 + lg < nblocks ? (sq[s * 2 + q] >> (8 * lg)) & 255u : 0u;
                const float sc = __uint_as_float(sb << 23);
                const unsigned wd[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const chunk_t op = open_fp4x8(wd[j], sc);
#pragma unroll
                    for (int tb = 0; tb < TBLK; ++tb)
                        Elem<E>::mma16(acc[tb], op, xs[(tb * 16 + li) * SC + ((s * 32 + q * 16 + lg * 4 + j) ^ li)]);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        }
    }
    // acc[tb][e] = D[weight row blk * 16 + lg * 4 + e][token tb * 16 + li]: token-major KiB tiles, as decode_stream_kernel's
    float4 *P4 = reinterpret_cast<float4 *>(set.P) + ((int64_t)(pblk * p.ks + slice) * TBLK) * 64 + li * 4 + lg;
#pragma unroll
    for (int tb = 0; tb < TBLK; ++tb)
        if (keep >> tb & 1u) P4[tb * 64] = make_float4(acc[tb][0], acc[tb][1], acc[tb][2], acc[tb][3]);
}

template <int TBLK, int SC>
constexpr size_t mx_stream_smem(int waves) {
    return (size_t)TBLK * 16 * SC * 16 + (size_t)waves * 2048;
}

template <int TBLK, int SC, bool X8>
hipError_t launch_t(const MxDecodeArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    MxDecodeArgs a = a0;
    const int w = a.d.waves;
    a.ext_groups = (a.d.nbe + w - 1) / w;
    long groups = 0;
    for (int i = 0; i < a.n; ++i) {
        a.w[i].group0 = (int32_t)groups;
        groups += a.ext_groups + (a.d.set[i].nbw + w - 1) / w;
    }
    const long grid = groups * a.d.ks;
    return launch_kernel(mx_decode_stream_kernel<TBLK, SC, X8>, dim3((unsigned)grid), dim3(w * 64), mx_stream_smem<TBLK, SC>(w), stream, timer, a);
}
template <int TBLK, int SC>
hipError_t init_t() {
    constexpr int smem = (int)mx_stream_smem<TBLK, SC>(kDecodeMaxWaves);
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(mx_decode_stream_kernel<TBLK, SC, false>), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == hipSuccess)
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(mx_decode_stream_kernel<TBLK, SC, true>), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    return e;
}
template <int TBLK>
hipError_t launch_b(const MxDecodeArgs &a, hipStream_t stream, const KernelTimer *timer) {
    if constexpr (TBLK <= kMxWideBlocks) {
        if (a.d.slice_chunks == 128)
            return a.Xq ? launch_t<TBLK, 128, true>(a, stream, timer) : launch_t<TBLK, 128, false>(a, stream, timer);
    }
    if (a.d.slice_chunks != 64) return hipErrorInvalidValue;
    return a.Xq ? launch_t<TBLK, 64, true>(a, stream, timer) : launch_t<TBLK, 64, false>(a, stream, timer);
}
template <int TBLK>
hipError_t init_b() {
    hipError_t e = init_t<TBLK, 64>();
    if constexpr (TBLK <= kMxWideBlocks) {
        if (e == hipSuccess) e = init_t<TBLK, 128>();
    }
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
          a.n <= kMaxGemmSets && d.slice_chunks > 0 && d.ks == (d.K / 8 + d.slice_chunks - 1) / d.slice_chunks && d.waves >= kDecodeMinWaves &&
          d.waves <= kDecodeMaxWaves && (d.X != nullptr || (a.Xq != nullptr && d.nbe == 0))))
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
