// Tiled product of a 4-bit backbone and 8-bit activations, both with a scale for every 32 values:
//
//     Y[row, n] = sum_k X[row, k] W[n, k]  (+ D[row, n] for rows with an adapter),   rounded once
//
// on the block-scaled matrix instructions: one 16x16x128 MFMA takes 128 values of 16 rows of W (e2m1) and of 16 rows of X
// (e4m3) with the scales of their blocks, so nothing is ever taken apart.  Of a 16-row operand of W, lane l holds block l / 16
// of row l % 16 (16 bytes); of X the 16-byte pieces l / 16 and 4 + l / 16 of the row's 128 bytes (measured: element e of lane
// group g is value 16 g + e for e < 16, 48 + 16 g + e behind); a scale operand is block l / 16's of row l % 16 for both.
#include "mx_kernels.h"

namespace lora {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ unsigned load_u32(const void *p) { return *(const __attribute__((address_space(1))) unsigned *)p; }

// LDS position (in 16-byte pieces) of piece c of row r: rows of X of 8 pieces, rows of W of 4, two to a line of 8.
__device__ __forceinline__ int x_at(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }
__device__ __forceinline__ int w_at(int r, int c) { return (r >> 1) * 8 + ((((r & 1) << 2) | c) ^ ((r >> 2) & 3)); }

template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64) void mx_gemm_kernel(MxGemmArgs p, int tiles_m, int tiles_n, int group_m) {
    constexpr int NT = WM * WN * 64;
    constexpr int WTM = BM / WM, WTN = BN / WN, NBT = WTM / 16, NBN = WTN / 16;
    constexpr int XL = BM * 8 / NT, WL = BN * 4 / NT;
    static_assert(XL * NT == BM * 8 && WL * NT == BN * 4 && BM + BN <= NT * 2 && NBN % 2 == 0, "tile and workgroup");
    __shared__ __attribute__((aligned(16))) chunk_t sX[BM * 8];
    __shared__ __attribute__((aligned(16))) chunk_t sW[BN * 4];
    __shared__ unsigned sS[BM + BN];
    __shared__ int srow[BM];
    __shared__ unsigned char use_d[BM];

    const int total = tiles_m * tiles_n;
    const int per_xcd = (total + 7) >> 3;
    const int lin = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (lin >= total) return;
    const int width = group_m * tiles_n;
    const int first_m = lin / width * group_m;
    const int gsz = min(tiles_m - first_m, group_m);
    const int pm = first_m + (lin % width) % gsz, pn = (lin % width) / gsz;
    int si = 0;
    while (si + 1 < p.n_sets && pn >= p.set[si + 1].tile0) ++si;
    const MxGemmSet g = p.set[si];
    const int m0 = pm * BM, n0 = (pn - g.tile0) * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn0 = (wave % WN) * WTN, wm0 = (wave / WN) * WTM;
    const int lr = lane & 15, lq = lane >> 4;
    if (p.plan.scalars[kScStatus] != 0) return;
    for (int r = tid; r < BM; r += NT) {
        const int t = min(m0 + r, p.T - 1);
        srow[r] = t;
        use_d[r] = g.D != nullptr && p.plan.row_adapter[t] >= 0;
    }
    const int nblocks = p.K / kMxBlock, KT = (nblocks + 3) / 4;
    f32x4_t acc[NBN][NBT];
#pragma unroll
    for (int nb = 0; nb < NBN; ++nb)
#pragma unroll
        for (int tb = 0; tb < NBT; ++tb) acc[nb][tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int kt = 0; kt < KT; ++kt) {
        chunk_t xr[XL], wr[WL];
        unsigned sr[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int idx = tid + i * NT, r = idx >> 3, c = kt * 8 + (idx & 7);
            xr[i] = load_chunk(p.Xq + (int64_t)min(m0 + r, p.T - 1) * p.ldxq + min(c, nblocks * 2 - 1) * 16);
            xr[i] = keep_if(c < nblocks * 2, xr[i]);
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int idx = tid + i * NT, r = idx >> 2, c = kt * 4 + (idx & 3);
            wr[i] = load_chunk(g.Wq + (int64_t)min(n0 + r, g.N - 1) * g.ldwq + min(c, nblocks - 1) * 16);
        }
        const unsigned live = nblocks - kt * 4 >= 4 ? ~0u : (1u << 8 * (nblocks - kt * 4)) - 1u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = tid + i * NT;
            if (r < BM)
                sr[i] = load_u32(p.Xs + (int64_t)min(m0 + r, p.T - 1) * p.ldxs + kt * 4) & live;
            else if (r < BM + BN)
                sr[i] = load_u32(g.Ws + (int64_t)min(n0 + r - BM, g.N - 1) * g.ldws + kt * 4) & live;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int idx = tid + i * NT;
            sX[x_at(idx >> 3, idx & 7)] = xr[i];
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int idx = tid + i * NT;
            sW[w_at(idx >> 2, idx & 3)] = wr[i];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (tid + i * NT < BM + BN) sS[tid + i * NT] = sr[i];
        __syncthreads();
        i32x8_t x[NBT];
        int xsc[NBT];
#pragma unroll
        for (int tb = 0; tb < NBT; ++tb) {
            const int r = wm0 + tb * 16 + lr;
            const chunk_t a = sX[x_at(r, lq)], b = sX[x_at(r, 4 + lq)];
            x[tb] = i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
            xsc[tb] = (int)(sS[r] >> (8 * lq));
        }
#pragma unroll
        for (int nb = 0; nb < NBN; ++nb) {
            const int r = wn0 + nb * 16 + lr;
            const chunk_t a = sW[w_at(r, lq)];
            const i32x8_t w{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
            const int wsc = (int)(sS[BM + r] >> (8 * lq));
#pragma unroll
            for (int tb = 0; tb < NBT; ++tb)
                acc[nb][tb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x[tb], acc[nb][tb], 4, 0, 0, wsc, 0, xsc[tb]);
        }
    }
    const int pc = n0 + wn0 + pair_column(lane);
    __bf16 *Y = static_cast<__bf16 *>(g.Y);
#pragma unroll
    for (int tb = 0; tb < NBT; ++tb) {
        const int t = wm0 + tb * 16 + lr;
        const bool ok = m0 + t < p.T, has = use_d[t] != 0;
#pragma unroll
        for (int i = 0; i < NBN / 2; ++i) {
            float v[8];
            pair_columns(acc[2 * i][tb], acc[2 * i + 1][tb], v);
            const int n = pc + i * 32;
            if (has) {
                float d[8];
                const float *src = g.D + (int64_t)srow[t] * g.ldd + min(n, (int)g.ldd - 8);
                const chunk_t a = load_chunk(src), b = load_chunk(src + 4);
                d[0] = __uint_as_float(a.x), d[1] = __uint_as_float(a.y), d[2] = __uint_as_float(a.z), d[3] = __uint_as_float(a.w);
                d[4] = __uint_as_float(b.x), d[5] = __uint_as_float(b.y), d[6] = __uint_as_float(b.z), d[7] = __uint_as_float(b.w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += d[e];
            }
            if (ok) store_columns(Y + (int64_t)srow[t] * g.ldy, n, g.N, v);
        }
    }
}

template <int BM, int BN, int WM, int WN>
hipError_t launch_t(const MxGemmArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    MxGemmArgs a = a0;
    const int tiles_m = (a.T + BM - 1) / BM;
    int tiles_n = 0;
    for (int i = 0; i < a.n_sets; ++i) {
        a.set[i].tile0 = tiles_n;
        tiles_n += (a.set[i].N + BN - 1) / BN;
    }
    const long total = (long)tiles_m * tiles_n;
    if (total <= 0) return hipSuccess;
    return launch_kernel(mx_gemm_kernel<BM, BN, WM, WN>, dim3((unsigned)((total + 7) / 8 * 8)), dim3(WM * WN * 64), 0, stream, timer, a, tiles_m,
                         tiles_n, 8);
}

}  // namespace

hipError_t init_mx_gemm_kernels() { return hipSuccess; }

hipError_t launch_mx_gemm(const MxGemmArgs &a, int variant, hipStream_t stream, const KernelTimer *timer) {
    if (!(a.T > 0 && a.K > 0 && a.K % kMxBlock == 0 && a.n_sets >= 1 && a.n_sets <= kMaxGemmSets && a.Xq && a.Xs)) return hipErrorInvalidValue;
    (void)variant;
    return launch_t<128, 128, 2, 2>(a, stream, timer);
}

}  // namespace lora
