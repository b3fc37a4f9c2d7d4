// The tile that the products in blocks and the products grouped by expert share.
//
// A workgroup makes BT rows (tokens, positions) x BN columns (output channels) of y.  Both operands lie with the summed dimension
// along their rows, so both are staged alike: 128 bytes of every row at a time (a slab: one block of 128 codes, or 64 values of 16
// bits), copied straight into LDS by direct-to-LDS loads while the slab before is multiplied.
//
// The weights are the first operand of the matrix instructions: a lane's sums then belong to ONE row of y per 16 rows, and
// the scale of a block, a_scale[row] * b_scale[128 columns], is one number per lane and 16 x 16 products.  A 16x16x128 product
// of codes is exactly one block; its four sums a lane are scaled and added in 32 bits (four multiply-adds beside a matrix
// instruction of 32 cycles).
//
// The 16 weight rows of a matrix operand are picked so that a lane ends up with eight neighbouring columns of y over two
// products (n = 32 (i/2) + 8 (r/4) + 4 (i%2) + r%4 for row r of product i): stores are 16 bytes wide.
//
// LDS: a row's eight 16-byte chunks are stored at chunk ^ key(row), with keys under which the 16 rows of an operand read from
// eight different places: no two lanes of a read that are served together meet in a bank.
#pragma once

#include "op_common.h"

namespace sc {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct MatmulArgs {
    const uint8_t* a;
    const uint8_t* b;
    const float* as;
    const float* bs;
    const float* bias;
    const int32_t* index;
    const int32_t* offsets;
    void* y;
    int M, N, E, a_rows;
    int kbytes;                              // bytes of a row that count
    int act;
    int64_t a_row, b_row, b_expert;          // bytes
    int64_t y_row;                           // elements
    int64_t as_row, bs_row, bs_expert;       // floats
};

constexpr int kSlab = 128;                   // bytes of a row that are staged at a time

// The 16 bytes of a row that begin at `at`, zeros behind the end of the row.
__device__ __forceinline__ v4i row_chunk(const uint8_t* row, int at, int kbytes)
{
    v4i v = {0, 0, 0, 0};
    if (at >= kbytes) return v;
    v = *reinterpret_cast<const v4i*>(row + at);
    const int have = kbytes - at;
    if (have < 16)
        for (int i = 0; i < 4; ++i) {
            const int h = have - 4 * i;
            v[i] = h <= 0 ? 0 : h >= 4 ? v[i] : v[i] & ((1 << (8 * h)) - 1);
        }
    return v;
}

// Eight codes as 16-bit floats (which hold every code).
__device__ __forceinline__ v8h widen8(int lo, int hi)
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float act_of(float z, int act)
{
    return act == SC_ACT_RELU ? activate<SC_ACT_RELU>(z) : act == SC_ACT_SILU ? activate<SC_ACT_SILU>(z) : z;
}

// Rows of group e: [lo, hi), whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int M, int& lo, int& hi)
{
    lo = min(max(offsets[e], 0), M);
    hi = max(lo, min(max(offsets[e + 1], 0), M));
}

// Group and rows of row tile `tile` (of BT rows) of all groups: every wave adds up the groups' tiles, 64 groups at a time.
// *total = row tiles in all, known where the tile is none of them (e = -1) and never smaller than tile + 1 else.
template <int BT> __device__ __forceinline__ int group_tile_count(const MatmulArgs& p)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int base = 0; base < p.E; base += 64) {
        int lo = 0, hi = 0;
        if (base + lane < p.E) group_rows(p.offsets, base + lane, p.M, lo, hi);
        int t = (hi - lo + BT - 1) / BT;
        for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
        total += t;
    }
    return __builtin_amdgcn_readfirstlane(total);
}

template <int BT> __device__ __forceinline__ bool find_group(const MatmulArgs& p, int tile, int& e, int& m0, int& hi_)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < p.E; base += 64) {
        int lo = 0, hi = 0;
        if (base + lane < p.E) group_rows(p.offsets, base + lane, p.M, lo, hi);
        const int t = (hi - lo + BT - 1) / BT;
        int upto = t;                                            // tiles of the groups up to this lane's
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        const uint64_t behind = __ballot(tile < upto);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            e = base + at;
            m0 = __builtin_amdgcn_readfirstlane(__shfl(lo + (tile - (upto - t)) * BT, at));
            hi_ = __builtin_amdgcn_readfirstlane(__shfl(hi, at));
            return true;
        }
        tile -= __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
    }
    return false;
}

// One 16-byte (or 4-byte) direct-to-LDS load a lane: lane i's bytes go to `lds` + i * width.  Written by hand so that the compiler does
// not make the reads of the other buffer wait for it; the caller waits on vmcnt itself.
typedef __attribute__((address_space(3))) void* lds_ptr_t;
template <int BYTES> __device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t off, uint32_t lds)
{
    uint32_t keep;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(off), "s"(base), "s"(lds) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(off), "s"(base), "s"(lds) : "memory");
}
template <int BYTES> __device__ __forceinline__ void to_lds_ptr(const uint8_t* src, uint32_t lds)
{
    uint32_t keep;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(src), "s"(lds) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(src), "s"(lds) : "memory");
}

__device__ __forceinline__ int token_key(int row) { return row & 7; }
__device__ __forceinline__ int weight_key(int row) { return (row & 3) | ((row >> 1) & 4); }

// BT x BN of y per workgroup, WT x WN waves.  AT: type of the operands, YT: of y.
template <int AT, int YT, bool GROUPED, int BT, int BN, int WT, int WN>
__global__ __launch_bounds__(WT * WN * 64, 2) void matmul_tile_kernel(MatmulArgs p)
{
    constexpr int W = WT * WN, TF = BT / WT / 16, NF = BN / WN / 16;    // waves; 16-row products of a wave along the rows / columns of y
    constexpr int AI = BT / 8 / W, BI = BN / 8 / W;                     // copies of 1 KB (eight rows) a wave makes of a slab
    constexpr bool CODES = AT == SC_ELEM_E4M3;
    constexpr int kStage = (BT + BN) * kSlab, kScales = CODES ? W * 64 * 4 : 0;
    static_assert(AI * 8 * W == BT && BI * 8 * W == BN && NF % 2 == 0, "tile");
    static_assert(!CODES || (BT + (BN + 127) / 128 <= W * 64), "one lane fetches a scale");
    __shared__ __align__(16) uint8_t lds[2 * (kStage + kScales)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntn = (p.N + BN - 1) / BN;

    // The place of this workgroup: neighbours in the order of launch go to different XCDs, so the ids are dealt out again such
    // that an XCD walks over neighbouring tiles, eight row tiles by eight column tiles at a time.
    int ntm = GROUPED ? group_tile_count<BT>(p) : (p.M + BT - 1) / BT;
    const int total = ntm * ntn;
    int id = blockIdx.x;
    if (id >= total) return;
    {
        const int each = total >> 3, more = total & 7, xcd = id & 7, at = id >> 3;
        id = xcd * each + min(xcd, more) + at;
    }
    const int band = id / (8 * ntn), inband = id - band * 8 * ntn, height = min(8, ntm - band * 8);
    const int tm = band * 8 + inband % height, tn = inband / height;
    int e = 0, m0 = tm * BT, hi = p.M;
    if constexpr (GROUPED)
        if (!find_group<BT>(p, tm, e, m0, hi)) return;
    const int n0 = tn * BN;
    const int rows = min(BT, hi - m0);

    // Where this lane's copies come from.  A copy is eight rows; lane i brings chunk (i & 7) ^ key of row i >> 3.  Rows beyond the last
    // one read the last one: what they add is not stored.
    const uint8_t* abase = p.a + (GROUPED ? 0 : (int64_t)m0 * p.a_row);
    const uint8_t* bbase = p.b + (GROUPED ? (int64_t)e * p.b_expert : 0) + (int64_t)n0 * p.b_row;
    uint32_t boff[BI], aoff[AI];
    const uint8_t* aptr[AI];
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        const int r = (wave + i * W) * 8 + (lane >> 3);
        boff[i] = (uint32_t)(min(r, p.N - 1 - n0) * p.b_row) + (((lane & 7) ^ weight_key(r)) << 4);
    }
#pragma unroll
    for (int i = 0; i < AI; ++i) {
        const int r = (wave + i * W) * 8 + (lane >> 3), chunk = ((lane & 7) ^ token_key(r)) << 4;
        if constexpr (GROUPED) {
            int m = m0 + min(r, rows - 1);
            if (p.index) m = p.index[m];
            // (an index that stands for zeros: any row that can be read; its sums are dropped)
            aptr[i] = (uint32_t)m < (uint32_t)p.a_rows ? p.a + m * p.a_row : p.b;
            aptr[i] += chunk;
        } else {
            aoff[i] = (uint32_t)(min(r, rows - 1) * p.a_row) + chunk;
        }
    }
    // Scales: BT of rows, then one for each 128 columns, one lane each.
    const uint8_t* sptr = nullptr;
    if constexpr (CODES) {
        const int j = tid;
        if (j < BT) {
            int m = m0 + min(j, rows - 1);
            if (GROUPED && p.index) m = p.index[m];
            sptr = reinterpret_cast<const uint8_t*>((uint32_t)m < (uint32_t)p.a_rows ? p.as + m * p.as_row : p.bs);
        } else {
            const int nb = min((n0 >> 7) + min(j - BT, (BN + 127) / 128 - 1), (p.N - 1) >> 7);
            sptr = reinterpret_cast<const uint8_t*>(p.bs + (GROUPED ? e * p.bs_expert : 0) + nb * p.bs_row);
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;

    // Slabs: a last, short one comes first (it is masked on its way through registers), then the whole ones in their order.
    const int whole = p.kbytes / kSlab, tail = p.kbytes % kSlab, slabs = whole + (tail != 0);
    auto stage = [&](int s, int buf) {       // whole slab s
        const uint32_t at = lds0 + buf * kStage;
#pragma unroll
        for (int i = 0; i < AI; ++i)
            if constexpr (GROUPED) to_lds_ptr<16>(aptr[i] + s * kSlab, at + (wave + i * W) * 1024);
            else to_lds<16>(abase + s * kSlab, aoff[i], at + (wave + i * W) * 1024);
#pragma unroll
        for (int i = 0; i < BI; ++i) to_lds<16>(bbase + s * kSlab, boff[i], at + BT * kSlab + (wave + i * W) * 1024);
        if constexpr (CODES) to_lds_ptr<4>(sptr + s * 4, lds0 + 2 * kStage + buf * kScales + wave * 256);
    };
    if (tail) {
        for (int i = 0; i < AI + BI; ++i) {
            const bool of_a = i < AI;
            const int j = of_a ? i : i - AI;
            const int r = (wave + j * W) * 8 + (lane >> 3);
            const int chunk = ((lane & 7) ^ (of_a ? token_key(r) : weight_key(r))) << 4;
            const uint8_t* row;
            if (of_a) {
                int m = m0 + min(r, rows - 1);
                if (GROUPED && p.index) m = p.index[m];
                row = (uint32_t)m < (uint32_t)p.a_rows ? p.a + m * p.a_row : p.b;
            } else {
                row = bbase + min(r, p.N - 1 - n0) * p.b_row;
            }
            *reinterpret_cast<v4i*>(lds + (of_a ? 0 : BT * kSlab) + (wave + j * W) * 1024 + lane * 16) = row_chunk(row + whole * kSlab, chunk, tail);
        }
        if constexpr (CODES) *reinterpret_cast<float*>(lds + 2 * kStage + tid * 4) = *reinterpret_cast<const float*>(sptr + whole * 4);
    } else {
        stage(0, 0);
    }

    const int wt = wave % WT, wn = wave / WT;
    const int c = lane & 15, q = lane >> 4;
    // This lane's places in a slab: token row c of a product, weight row 8 (c/4) + c%4 of a pair of products.
    const int trow = wt * (TF * 16) + c, wrow = wn * (NF * 16) + (c >> 2) * 8 + (c & 3);
    v4f acc[NF][TF] = {};
    for (int it = 0; it < slabs; ++it) {
        const int buf = it & 1;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (it + 1 < slabs) stage(tail ? it : it + 1, buf ^ 1);
        const uint8_t* A = lds + buf * kStage;
        const uint8_t* Bm = A + BT * kSlab;
        const float* S = reinterpret_cast<const float*>(lds + 2 * kStage + buf * kScales);
        v4i t[TF][2];
        float sc[TF];
#pragma unroll
        for (int j = 0; j < TF; ++j) {
            const int r = trow + 16 * j;
#pragma unroll
            for (int h = 0; h < 2; ++h) t[j][h] = *reinterpret_cast<const v4i*>(A + r * kSlab + (((2 * q + h) ^ token_key(r)) << 4));
            if constexpr (CODES) sc[j] = S[r] * S[BT + (wn * NF * 16) / 128];
        }
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int r = wrow + (i >> 1) * 32 + (i & 1) * 4;
            v4i w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) w[h] = *reinterpret_cast<const v4i*>(Bm + r * kSlab + (((2 * q + h) ^ weight_key(r)) << 4));
#pragma unroll
            for (int j = 0; j < TF; ++j) {
                if constexpr (CODES && YT == SC_ELEM_F32) {
                    v4f d = {0, 0, 0, 0};
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(w[h][2 * u], w[h][2 * u + 1]), widen8(t[j][h][2 * u], t[j][h][2 * u + 1]), d, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] += sc[j] * d[v];
                } else if constexpr (CODES) {
                    const v8i x = __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const v8i z = __builtin_shufflevector(t[j][0], t[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const v4f d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, z, v4f{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] += sc[j] * d[v];
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if constexpr (AT == SC_ELEM_F16)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w[h]), __builtin_bit_cast(v8h, t[j][h]), acc[i][j], 0, 0, 0);
                        else
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, w[h]), __builtin_bit_cast(v8b, t[j][h]), acc[i][j], 0, 0, 0);
                }
            }
        }
    }

    // y: a lane has eight neighbouring columns per pair of products.
    const bool wide = (reinterpret_cast<uintptr_t>(p.y) & 15) == 0 && (p.y_row * (int64_t)sizeof(Elem<YT>)) % 16 == 0;
    const float* bias = p.bias ? p.bias + (GROUPED ? (int64_t)e * p.N : 0) : nullptr;
#pragma unroll
    for (int j = 0; j < TF; ++j) {
        const int r = wt * (TF * 16) + 16 * j + c;
        if (r >= rows) continue;
        bool zero = false;
        if constexpr (GROUPED) zero = p.index && (uint32_t)p.index[m0 + r] >= (uint32_t)p.a_rows;
        Elem<YT>* y = static_cast<Elem<YT>*>(p.y) + (int64_t)(m0 + r) * p.y_row;
#pragma unroll
        for (int i = 0; i < NF; i += 2) {
            const int n = n0 + wn * (NF * 16) + (i >> 1) * 32 + q * 8;
            if (n >= p.N) continue;
            typedef Elem<YT> v8y __attribute__((ext_vector_type(8)));
            v8y out;
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                float z = zero ? 0.0f : acc[i + (v >> 2)][j][v & 3];
                if (bias) z += bias[min(n + v, p.N - 1)];
                out[v] = (Elem<YT>)act_of(z, p.act);
            }
            if (wide && n + 8 <= p.N) {
                *reinterpret_cast<v8y*>(y + n) = out;
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    if (n + v < p.N) y[n + v] = out[v];
            }
        }
    }
}

}  // namespace sc
