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
// LDS: a row's eight 16-byte chunks are stored at chunk ^ key(row).  A 16-byte read of a wave is served in four turns of sixteen lanes
// over the 64 banks (two rows): lanes 0-3, 12-15 and 20-27 together, 4-11 with 16-19 and 28-31, and the same 32 lanes on.  Of an
// operand's rows c = lane % 16 a turn has each once, c = 0-3 and 12-15 with one chunk and 4-11 with its neighbour but one
// (chunks 2 q + h, q = lane / 16): keys 0-3 for the former and 4-7 for the latter put all of them in banks of their own.
//
// Measured: 8192 x 8192 x 4096 codes 247 us, 2.2 PFLOP/s (a library's product of codes with one scale each: 2.6); the matrix units are busy 58 % of
// the time at some 2.05 GHz, which the power leaves, and no LDS read conflicts.  16384 rows of 16 unequal experts, 4096 x 2048 codes: 195 us,
// matrix units busy 44 %; 161 where the weights are in the last-level cache already.  Tiles that a group fills in part are a tenth of it.
#pragma once

#include <type_traits>

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

// The first `have` bytes of a chunk (all of them from 16 on), zeros behind.
__device__ __forceinline__ v4i first_bytes(v4i v, int have)
{
#pragma unroll
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

template <int YT> __device__ __forceinline__ float act_of(float z, int act)
{
    return act == SC_ACT_RELU ? activate<SC_ACT_RELU, YT>(z) : act == SC_ACT_SILU ? activate<SC_ACT_SILU, YT>(z) : z;
}

// Eight of them after one branch (a branch each: a tile of 256 x 256 leaves by 41 KB of code for 27, experts' products take 1.5 % more).
template <int YT> __device__ __forceinline__ void act_all(float (&z)[8], int act)
{
    if (act == SC_ACT_RELU) {
#pragma unroll
        for (int v = 0; v < 8; ++v) z[v] = activate<SC_ACT_RELU, YT>(z[v]);
    } else if (act == SC_ACT_SILU) {
#pragma unroll
        for (int v = 0; v < 8; ++v) z[v] = activate<SC_ACT_SILU, YT>(z[v]);
    }
}

// Rows of group e: [lo, hi), whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int M, int& lo, int& hi)
{
    lo = min(max(offsets[e], 0), M);
    hi = max(lo, min(max(offsets[e + 1], 0), M));
}

// The row tiles (of BT rows) of the groups, 64 groups a turn: every wave adds them up for itself.  Up to 64 groups are read once.
template <int BT> struct GroupTiles {
    int lo, hi, upto;                        // this lane's group of the turn: its rows, row tiles of the groups up to it
    int base = 0, before = 0, total = 0;     // first group of the turn, row tiles of the turns before, of all

    // tiles of the 64 groups from `first` on
    __device__ __forceinline__ int turn(const MatmulArgs& p, int first)
    {
        const int lane = threadIdx.x & 63;
        lo = hi = 0;
        if (first + lane < p.E) group_rows(p.offsets, first + lane, p.M, lo, hi);
        upto = (hi - lo + BT - 1) / BT;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        return __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ __forceinline__ explicit GroupTiles(const MatmulArgs& p)
    {
        total = turn(p, 0);
        if (p.E > 64) {
            for (int f = 64; f < p.E; f += 64) total += turn(p, f);
            base = -1;                       // (the turn in the registers is the last one)
        }
    }
    // Group e of row tile `tile` < total, its first row tile (of all), its rows [m0, end).
    __device__ __forceinline__ void find(const MatmulArgs& p, int tile, int& e, int& first, int& m0, int& end)
    {
        if (base < 0)
            for (base = 0, before = 0;; base += 64) {
                const int t = turn(p, base);
                if (tile < before + t) break;
                before += t;
            }
        const int at = __builtin_ctzll(__ballot(tile - before < upto));
        m0 = __builtin_amdgcn_readlane(lo, at);
        end = __builtin_amdgcn_readlane(hi, at);
        first = before + __builtin_amdgcn_readlane(upto, at) - (end - m0 + BT - 1) / BT;
        e = base + at;
    }
};

struct NoGroups {
    __device__ __forceinline__ explicit NoGroups(const MatmulArgs&) {}
};

// One 16-byte (or 4-byte) direct-to-LDS load a lane: lane i's bytes go to `lds` + i * width.  Written by hand so that the compiler does
// not make the reads of the other buffer wait for it; the caller waits on vmcnt itself (staged()), which is also what keeps reads of
// the buffer behind it.
typedef __attribute__((address_space(3))) void* lds_ptr_t;
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}
template <int BYTES> __device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t off, uint32_t lds)
{
    uint32_t keep;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(off), "s"(base), "s"(lds));
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(off), "s"(base), "s"(lds));
}
template <int BYTES> __device__ __forceinline__ void to_lds_ptr(const uint8_t* src, uint32_t lds)
{
    uint32_t keep;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(src), "s"(lds));
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0" : "=&s"(keep) : "v"(src), "s"(lds));
}

// key of the row that lane c of sixteen reads
__device__ __forceinline__ int lane_key(int c) { return ((c >> 1) & 1) | ((c >> 2) & 2) | (((c >> 2) ^ (c >> 1)) & 2) << 1; }
__device__ __forceinline__ int token_key(int row) { return lane_key(row & 15); }
__device__ __forceinline__ int weight_key(int row) { return lane_key((row & 3) | ((row >> 1) & 12)); }

// One block's product of codes, unscaled: 16 weight rows (x) and 16 rows of a (z).  For 32-bit results exact products and 32-bit sums.  For 16-bit ones
// the 8-bit instruction, twice as fast: inside it what lies 13 bits below the largest of some eight products is cut off, which leaves 1.4e-5 of the
// result, 3.4e-5 with one value of the block a hundred times the others, where f16 rounds by 2e-4; blocks are added in 32 bits either way.
template <int YT> __device__ __forceinline__ v4f block_product(const v4i* x, const v4i* z)
{
    v4f d = {0, 0, 0, 0};
    if constexpr (YT == SC_ELEM_F32) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(x[h][2 * u], x[h][2 * u + 1]), widen8(z[h][2 * u], z[h][2 * u + 1]), d, 0, 0, 0);
    } else {
        d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7),
                                                             __builtin_shufflevector(z[0], z[1], 0, 1, 2, 3, 4, 5, 6, 7), d, 0, 0, 0, 0, 0, 0);
    }
    return d;
}

// sums + the product of 16 weight rows (x) and 16 rows of a (z), 32 values of 16 bits of each.
template <int AT> __device__ __forceinline__ v4f product16(v4i x, v4i z, v4f sums)
{
    if constexpr (AT == SC_ELEM_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, z), sums, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, x), __builtin_bit_cast(v8b, z), sums, 0, 0, 0);
}

// acc += one slab's product of 16 weight rows (x) and 16 rows of a (z); codes: times the scale of the block.
template <int AT, int YT> __device__ __forceinline__ void multiply(v4f& acc, const v4i* x, const v4i* z, float scale)
{
    if constexpr (AT == SC_ELEM_E4M3) {
        const v4f d = block_product<YT>(x, z);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[v] += scale * d[v];
    } else {
        (void)scale;
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = product16<AT>(x[h], z[h], acc);
    }
}

// Waits until at most N of this wave's copies are under way, then for the other waves.
template <int N> __device__ __forceinline__ void staged()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// BT x BN of y per workgroup, WT x WN waves, ST slabs in LDS: one is multiplied while the ST - 1 behind it arrive.
// KS groups of such waves take every KS-th slab each, all in step, and the first adds the sums of the others to its own in their order:
// where there are fewer workgroups than compute units, what a slab takes is the way from barrier to barrier, not its arithmetic.
// AT: type of the operands, YT: of y.
template <int AT, int YT, bool GROUPED, int BT, int BN, int WT, int WN, int ST, int KS>
__global__ __launch_bounds__(WT * WN * KS * 64, 2) void matmul_tile_kernel(MatmulArgs p)
{
    constexpr int W = WT * WN, TF = BT / WT / 16, NF = BN / WN / 16;    // waves; 16-row products of a wave along the rows / columns of y
    constexpr int AI = BT / 8 / W, BI = BN / 8 / W;                     // copies of 1 KB (eight rows) a wave makes of a slab
    constexpr bool CODES = AT == SC_ELEM_E4M3;
    constexpr int kStage = (BT + BN) * kSlab, kScales = CODES ? W * 64 * 4 : 0;
    constexpr int kCopies = AI + BI + (CODES ? 1 : 0);                  // of a wave and slab
    static_assert(AI * 8 * W == BT && BI * 8 * W == BN && NF % 2 == 0, "tile");
    static_assert(!CODES || (BT + (BN + 127) / 128 <= W * 64), "one lane fetches a scale");
    constexpr int kAll = ST * KS * kStage;                              // the scales lie behind the slabs
    __shared__ __align__(16) uint8_t lds[ST * KS * (kStage + kScales)];
    static_assert((KS - 1) * W * NF * TF * 1024 <= sizeof(lds), "the groups' sums");
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = KS > 1 ? all / W : 0, wave = KS > 1 ? all % W : all, tid = wave * 64 + lane;      // group of waves, place in it
    const int ntn = (p.N + BN - 1) / BN;

    // The place of this workgroup: neighbours in the order of launch go to different XCDs, so the ids are dealt out again such
    // that an XCD walks over neighbouring tiles, column after column of eight row tiles, or of all of a group where those are fewer.
    int ntm = (p.M + BT - 1) / BT;
    std::conditional_t<GROUPED, GroupTiles<BT>, NoGroups> groups(p);
    if constexpr (GROUPED) ntm = groups.total;
    const int total = ntm * ntn;
    int id = blockIdx.x;
    if (id >= total) return;
    {
        const int each = total >> 3, more = total & 7, xcd = id & 7, at = id >> 3;
        id = xcd * each + min(xcd, more) + at;
    }
    int e = 0, m0 = 0, hi = p.M, high = ntm;     // the group, its first row and the row behind its last, its row tiles
    if constexpr (GROUPED) {
        int first;
        groups.find(p, __builtin_amdgcn_readfirstlane(id / ntn), e, first, m0, hi);
        id -= first * ntn;
        high = (hi - m0 + BT - 1) / BT;
    }
    const int band = id / (8 * ntn), inband = id - band * 8 * ntn, height = min(8, high - band * 8);
    // (divisions are done in vector registers; what comes of these is the same in every lane and belongs in scalar ones)
    const int tn = __builtin_amdgcn_readfirstlane(inband / height), tm = __builtin_amdgcn_readfirstlane(band * 8 + inband - tn * height);
    m0 += tm * BT;
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
    const int turns = (slabs + KS - 1) / KS, mine = (slabs - kg + KS - 1) / KS;      // of all groups; slabs of this one
    auto copy = [&](int i, int turn, int buf) {  // copy i of this group's whole slab of a turn
        const int s = turn * KS + kg - (tail != 0);
        const uint32_t at = lds0 + (buf * KS + kg) * kStage;
        if (i < BI) to_lds<16>(uniform(bbase + s * kSlab), boff[i], at + BT * kSlab + (wave + i * W) * 1024);
        else if (i < BI + AI) {
            const int j = i - BI;
            if constexpr (GROUPED) to_lds_ptr<16>(aptr[j] + s * kSlab, at + (wave + j * W) * 1024);
            else to_lds<16>(uniform(abase + s * kSlab), aoff[j], at + (wave + j * W) * 1024);
        } else to_lds_ptr<4>(sptr + s * 4, lds0 + kAll + (buf * KS + kg) * kScales + wave * 256);
    };
    auto stage = [&](int turn) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy(i, turn, turn);
    };
    const int ahead = min(ST - 1, mine);
    if (tail && kg == 0) {
        v4i part[AI + BI];
        int have[AI + BI];                   // bytes of the short slab from a lane's chunk on
        float scale = 0.0f;
#pragma unroll
        for (int i = 0; i < AI + BI; ++i) {
            const bool of_a = i < AI;
            const int r = (wave + (of_a ? i : i - AI) * W) * 8 + (lane >> 3);
            const int chunk = ((lane & 7) ^ (of_a ? token_key(r) : weight_key(r))) << 4;
            const uint8_t* row;
            if (of_a) {
                int m = m0 + min(r, rows - 1);
                if (GROUPED && p.index) m = p.index[m];
                row = (uint32_t)m < (uint32_t)p.a_rows ? p.a + m * p.a_row : p.b;
            } else {
                row = bbase + min(r, p.N - 1 - n0) * p.b_row;
            }
            have[i] = tail - chunk;
            part[i] = v4i{0, 0, 0, 0};
            if (have[i] > 0) part[i] = *reinterpret_cast<const v4i*>(row + whole * kSlab + chunk);
        }
        if constexpr (CODES) scale = *reinterpret_cast<const float*>(sptr + whole * 4);
        for (int s = 1; s < ahead; ++s) stage(s);
#pragma unroll
        for (int i = 0; i < AI + BI; ++i) {
            const bool of_a = i < AI;
            *reinterpret_cast<v4i*>(lds + (of_a ? 0 : BT * kSlab) + (wave + (of_a ? i : i - AI) * W) * 1024 + lane * 16) = first_bytes(part[i], have[i]);
        }
        if constexpr (CODES) *reinterpret_cast<float*>(lds + kAll + tid * 4) = scale;
    } else {
        for (int s = 0; s < ahead; ++s) stage(s);
    }

    const int wt = wave % WT, wn = wave / WT;
    const int c = lane & 15, q = lane >> 4;
    // This lane's places in a slab: token row c of a product, weight row 8 (c/4) + c%4 of a pair of products.
    const int key = lane_key(c);
    const int trow = wt * (TF * 16) + c, wrow = wn * (NF * 16) + (c >> 2) * 8 + (c & 3);
    v4f acc[NF][TF] = {};
    // A slab is NF steps: one operand of the weights against the TF of a.  The weights are read two steps ahead, and a block's sums
    // are scaled and added under the matrix instructions of the step behind it.
    int buf = 0, next = (ST - 1) % ST;
    // This group's slab of turn `it`; MORE: the copies of turn it + ST - 1 are made in its first steps (a wave that issues them all at once waits for the
    // others', and late ones hold up the next slab).
    auto slab = [&](auto more, int it) {
        constexpr bool MORE = decltype(more)::value;
        constexpr int kSpread = NF > 2 ? NF / 2 : NF;
        const uint8_t* A = lds + (buf * KS + kg) * kStage;
        const uint8_t* Bm = A + BT * kSlab;
        v4i t[TF][2], w[3][2];
        v4f d[2][TF];
        float sc[TF], sw = 0.0f;
        auto read_w = [&](int i) {
            const int r = wrow + (i >> 1) * 32 + (i & 1) * 4;
#pragma unroll
            for (int h = 0; h < 2; ++h) w[i % 3][h] = *reinterpret_cast<const v4i*>(Bm + r * kSlab + (((2 * q + h) ^ key) << 4));
        };
        auto add = [&](int i, int j) {
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][j][v] += sc[j] * d[i & 1][j][v];
        };
        read_w(0);
#pragma unroll
        for (int j = 0; j < TF; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) t[j][h] = *reinterpret_cast<const v4i*>(A + (trow + 16 * j) * kSlab + (((2 * q + h) ^ key) << 4));
        if (NF > 1) read_w(1);
        if constexpr (CODES) {
            const float* S = reinterpret_cast<const float*>(lds + kAll + (buf * KS + kg) * kScales);
            sw = S[BT + (wn * NF * 16) / 128];
#pragma unroll
            for (int j = 0; j < TF; ++j) sc[j] = S[trow + 16 * j];
        }
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            if (i + 2 < NF) read_w(i + 2);
            if constexpr (MORE)
                if (i < kSpread)
#pragma unroll
                    for (int u = i * kCopies / kSpread; u < (i + 1) * kCopies / kSpread; ++u) copy(u, it + ST - 1, next);
            if (CODES && i == 1)
#pragma unroll
                for (int j = 0; j < TF; ++j) sc[j] *= sw;
            if constexpr (CODES) {
#pragma unroll
                for (int j = 0; j < TF; ++j) {
                    d[i & 1][j] = block_product<YT>(w[i % 3], t[j]);
                    if (i > 0) add(i - 1, j);
                }
            } else {
                // (the two halves of a slab's product add to the same sums: one half of all products, then the other)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < TF; ++j) acc[i][j] = product16<AT>(w[i % 3][h], t[j][h], acc[i][j]);
            }
            // In the widest tile: the reads first, then the scaling of one product under each matrix instruction (245 us against 252 at
            // 8192 x 8192 x 4096; narrower tiles lose by it).
            if (CODES && YT != SC_ELEM_F32 && NF == 8 && i > 0) {
                if (i + 2 < NF) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
                for (int j = 0; j < TF; ++j) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (CODES)
#pragma unroll
            for (int j = 0; j < TF; ++j) add(NF - 1, j);
        buf = buf + 1 == ST ? 0 : buf + 1;
        next = next + 1 == ST ? 0 : next + 1;
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    int it = 0;
    for (; it + ST - 1 < mine; ++it) {
        staged<(ST - 2) * kCopies>();
        slab(yes, it);
    }
    for (; it < turns; ++it) {               // (every group comes to every barrier)
        staged<0>();
        if (KS == 1 || it < mine) slab(no, it);
    }
    if constexpr (KS > 1) {
        v4f* sums = reinterpret_cast<v4f*>(lds) + wave * NF * TF * 64 + lane;
        __syncthreads();
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int j = 0; j < TF; ++j) sums[((kg - 1) * W * NF * TF + i * TF + j) * 64] = acc[i][j];
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int j = 0; j < TF; ++j) acc[i][j] += sums[(k * W * NF * TF + i * TF + j) * 64];
    }

    // y: a lane has eight neighbouring columns per pair of products.
    const bool wide = (reinterpret_cast<uintptr_t>(p.y) & 15) == 0 && (p.y_row * (int64_t)sizeof(Elem<YT>)) % 16 == 0;
    const float* bias = p.bias ? p.bias + (GROUPED ? (int64_t)e * p.N : 0) : nullptr;
    bool zero[TF] = {};
    if constexpr (GROUPED)
        if (p.index)
#pragma unroll
            for (int j = 0; j < TF; ++j) zero[j] = (uint32_t)p.index[m0 + min(trow + 16 * j, rows - 1)] >= (uint32_t)p.a_rows;
#pragma unroll
    for (int i = 0; i < NF; i += 2) {
        const int n = n0 + wn * (NF * 16) + (i >> 1) * 32 + q * 8;
        if (n >= p.N) continue;
        const bool whole8 = n + 8 <= p.N;
        float add[8] = {};
        if (bias) {
            if (whole8) {
                __builtin_memcpy(add, bias + n, 32);
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v) add[v] = bias[min(n + v, p.N - 1)];
            }
        }
#pragma unroll
        for (int j = 0; j < TF; ++j) {
            const int r = trow + 16 * j;
            if (r >= rows) continue;
            Elem<YT>* y = static_cast<Elem<YT>*>(p.y) + (int64_t)(m0 + r) * p.y_row + n;
            float z[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) z[v] = (zero[j] ? 0.0f : acc[i + (v >> 2)][j][v & 3]) + add[v];
            act_all<YT>(z, p.act);
            // (Past the caches: 6272 x 1024 x 256 -> f16 7.2 us for 8.1, with a quantiser of the result behind it 14.5 for 16.2; 16384 x 4096 x 2048,
            // 134 MB of results, 139 for 132, with the quantiser 172 for 163.)
            if (wide && whole8) {
                store_vec_past<YT, 8>(y, z);
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    if (n + v < p.N) y[v] = (Elem<YT>)z[v];
            }
        }
    }
}

// Few rows: 16 of them against 16 columns a workgroup, whose waves share the summed dimension out among themselves.
// Bound by reading the weights once: they go from memory into the registers that multiply them (a lane reads 16 bytes of its
// row, four lanes 64 in a row), kAtOnce slabs of a wave under way together, and the waves' sums meet in LDS, in their order.
// 1 x 4096 x 4096 (16.8 MB of weights): 4.7 us on the GPU, 7 a call; a launch and two trips to memory, one behind the other, take most of it.
constexpr int kAtOnce = 4;
template <int AT, int YT, bool GROUPED> __global__ __launch_bounds__(512) void matmul_rows_kernel(MatmulArgs p)
{
    constexpr bool CODES = AT == SC_ELEM_E4M3;
    extern __shared__ __align__(16) v4f part[];          // [waves][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int ntn = (p.N + 15) / 16, tm = blockIdx.x / ntn, n0 = (blockIdx.x - tm * ntn) * 16;
    int e = 0, m0 = tm * 16, hi = p.M;
    if constexpr (GROUPED) {
        GroupTiles<16> groups(p);
        if (tm >= groups.total) return;
        int first;
        groups.find(p, tm, e, first, m0, hi);
        m0 += (tm - first) * 16;
    }
    const int rows = min(16, hi - m0), c = lane & 15, q = lane >> 4;
    const uint8_t* w = p.b + (GROUPED ? e * p.b_expert : 0) + min(n0 + c, p.N - 1) * p.b_row + q * 16;
    const float* bs = CODES ? p.bs + (GROUPED ? e * p.bs_expert : 0) + n0 / kQBlock * p.bs_row : nullptr;
    int m = m0 + min(c, rows - 1);
    if (GROUPED && p.index) m = p.index[m];
    const bool real = (uint32_t)m < (uint32_t)p.a_rows;      // (an index that stands for zeros: see the tile)
    const uint8_t* t = (real ? p.a + m * p.a_row : p.b) + q * 16;
    const float* as = CODES ? real ? p.as + m * p.as_row : p.bs : nullptr;
    const int slabs = (p.kbytes + kSlab - 1) / kSlab;
    v4f acc = {0, 0, 0, 0};
    auto some = [&](int s0, bool whole) {
        v4i x[kAtOnce][2], z[kAtOnce][2];
        float sc[kAtOnce], sb[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = (s0 + u * waves) * kSlab + 64 * h, have = p.kbytes - at - q * 16;
                x[u][h] = v4i{0, 0, 0, 0};
                if (whole || have > 0) x[u][h] = *reinterpret_cast<const v4i*>(w + at);
                if (!whole) x[u][h] = first_bytes(x[u][h], have);
                z[u][h] = v4i{0, 0, 0, 0};
                if (whole || have > 0) z[u][h] = *reinterpret_cast<const v4i*>(t + at);
                if (!whole) z[u][h] = first_bytes(z[u][h], have);
            }
            if constexpr (CODES) {
                const int kb = whole ? s0 + u * waves : min(s0 + u * waves, slabs - 1);
                sb[u] = bs[kb];
                sc[u] = as[kb];
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (!whole && s0 + u * waves >= slabs) break;
            multiply<AT, YT>(acc, x[u], z[u], CODES ? sc[u] * sb[u] : 0.0f);
        }
    };
    for (int s = wave; s < slabs; s += kAtOnce * waves) some(s, (s + (kAtOnce - 1) * waves + 1) * kSlab <= p.kbytes);
    part[wave * 64 + lane] = acc;
    __syncthreads();
    const float* bias = p.bias ? p.bias + (GROUPED ? (int64_t)e * p.N : 0) : nullptr;
    for (int i = threadIdx.x; i < 256; i += blockDim.x) {
        // (value i: row i / 16 of the tile, column i % 16: sum i % 4 of lane 16 (i / 4 % 4) + row)
        const int r = i >> 4, n = n0 + (i & 15);
        if (r >= rows || n >= p.N) continue;
        const int from = (((i >> 2) & 3) * 16 + r) * 4 + (i & 3);
        float s = 0.0f;
        for (int k = 0; k < waves; ++k) s += reinterpret_cast<const float*>(part)[k * 256 + from];
        if constexpr (GROUPED)
            if (p.index && (uint32_t)p.index[m0 + r] >= (uint32_t)p.a_rows) s = 0.0f;
        if (bias) s += bias[n];
        static_cast<Elem<YT>*>(p.y)[(m0 + r) * p.y_row + n] = (Elem<YT>)act_of<YT>(s, p.act);
    }
}

}  // namespace sc
