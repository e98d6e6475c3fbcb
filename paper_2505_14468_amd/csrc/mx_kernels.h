// Host-side launch interface between mx_api.hiph and the kernels on block-scaled formats.
#pragma once
#include "kernels.h"

namespace lora {

constexpr int kMxBlock = 32;
constexpr int kMxPieces = 4;               // of 64 x 8 values that a wave of the conversions takes: that many loads in flight
constexpr int kMxStrip = kMxPieces * 512;  // (rows x strips of a conversion stay below 2^31)
enum MxFormat { kMxE2M1 = 0, kMxE4M3 = 1 };

struct MxConvertArgs {
    const void *src;  // quantize: values; dequantize: codes
    int64_t lds;      // elements (values) or bytes (codes) from row to row
    void *dst;        // the other of the two
    int64_t ldd;
    unsigned char *scales;  // written by quantize, read by dequantize
    int64_t ldsc;
    int64_t rows;
    int32_t K;
    int32_t strips;   // pieces of a row that a wave takes (set by the launcher)
};
hipError_t launch_mx_quantize(const MxConvertArgs &a, int dtype, int format, hipStream_t stream, const KernelTimer *timer);
hipError_t launch_mx_dequantize(const MxConvertArgs &a, int dtype, int format, hipStream_t stream, const KernelTimer *timer);

struct RmsNormArgs {
    const void *X;
    int64_t ldx;
    const void *R;  // null: none
    int64_t ldr;
    const void *gamma;
    void *H;        // null: none
    int64_t ldh;
    void *Y;        // null: none
    int64_t ldy;
    unsigned char *codes;  // null: none
    int64_t ldc;
    unsigned char *scales;
    int64_t ldsc;
    int64_t rows;
    int32_t K;
    float eps;
};
hipError_t launch_rms_norm(const RmsNormArgs &a, int dtype, hipStream_t stream, const KernelTimer *timer);

// Decode-sized batches: the streaming launch of the decode path on 4-bit weights; the second launch is the decode path's own.
struct MxDecodeSet {
    const unsigned char *Wq;
    int64_t ldwq;
    const unsigned char *Ws;
    int64_t ldws;
    int32_t group0;  // first group of workgroups of this projection (set by the launcher)
    int32_t pad_;
};
struct MxDecodeArgs {
    DecodeArgs d;                // set[0 .. n) in use whatever n_sets says; ks counts slices of slice_chunks, ks_ext those of 64
    const unsigned char *Xq;     // null: d.X
    int64_t ldxq;
    const unsigned char *Xs;
    int64_t ldxs;
    int32_t n;                   // projections
    int32_t ext_groups;          // groups of workgroups for extension rows, per projection (set by the launcher)
    int32_t ext_wgs;             // workgroups for them, which come first (set by the launcher)
    MxDecodeSet w[kMaxGemmSets];
};
// Slices of 64 or 128 chunks, the longer as far as X's fits into 128 KB of LDS (16 bytes a row and chunk, or 8).  Workgroups of at least
// eleven waves where X on its way to LDS would take more registers than twelve leave (168; 64 rows 4096 -> 11008 with seven
// of them spilled: 19.2 us, 16.0 without).
constexpr int kMxMostChunks = 128;
constexpr int mx_fewest_waves(int tblk, int slice_chunks) { return tblk >= 7 || (slice_chunks == 128 && tblk >= 4) ? 11 : kDecodeMinWaves; }
hipError_t init_mx_decode_kernels();
hipError_t launch_mx_decode_stream(const MxDecodeArgs &a, int tblk, hipStream_t stream, const KernelTimer *timer);

// More rows: tiles on 4-bit weights and 8-bit activations.
enum MxTileVariant { kMxTile256x256 = 0, kMxTile128x256 = 1, kMxTile128x128 = 2, kMxTileMixed = 3, kMxTileCount };  // (mixed: 256x256, and 128x256 for the last rows)
struct MxGemmSet {
    const unsigned char *Wq;
    int64_t ldwq;
    const unsigned char *Ws;
    int64_t ldws;
    void *Y;
    int64_t ldy;
    const void *V;         // [T, r_max] bf16, original row order (null: no adapters)
    const void *const *B;  // device table (null: no adapters, or all of the adapter term comes in D)
    const float *D;        // adapter term in fp32, [T, ldd], rows with an adapter only (null: none)
    int64_t ldd;
    int32_t long_rows;     // > 0: D holds the term of segments shorter than this, the kernel computes the others'
    int32_t N;
    int32_t tile0;         // first column tile (set by the launcher)
    int32_t pad_;
};
struct MxGemmArgs {
    PlanView plan;
    const unsigned char *Xq;
    int64_t ldxq;
    const unsigned char *Xs;
    int64_t ldxs;
    int32_t T, K;
    int32_t r_max;
    int32_t parts;        // 1, or 2: X is the sum of two sets of values, part_bytes (a multiple of 512, zeros past K) and
    int32_t part_bytes;   // part_scales apart in a row
    int32_t part_scales;
    // > 1: the contraction axis in stretches of chunk_blocks blocks (a multiple of 16); one projection, no adapter term here;
    // partial sums to P[s][row][n], rows ldp floats long (launch_splitk_reduce sums them)
    int32_t split_k;
    int32_t chunk_blocks;
    float *P;
    int64_t ldp;
    int32_t n_sets;
    int32_t pad_;
    MxGemmSet set[kMaxGemmSets];
};
hipError_t init_mx_gemm_kernels();
hipError_t launch_mx_gemm(const MxGemmArgs &a, int variant, hipStream_t stream, const KernelTimer *timer);

// bf16 rows as the sum of two sets of 8-bit values (MxGemmArgs::parts == 2): codes [rows, 2 part_bytes], scales [rows, 2 part_scales].
struct MxSplitArgs {
    const void *X;
    int64_t ldx;
    unsigned char *codes;
    unsigned char *scales;
    int32_t rows, K;
    int32_t part_bytes, part_scales;
    int32_t strips;  // set by the launcher
};
hipError_t launch_mx_split(const MxSplitArgs &a, hipStream_t stream, const KernelTimer *timer);

}  // namespace lora
