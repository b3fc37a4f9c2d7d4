// Low-rank adapters of many requests beside a projection that they share (sparse_conv_adapters):
//     y[t] = base[t] + scale[e] (x[t] A_e^T) B_e^T      for the rows t of group e.
//
// Two launches, each in a form for few rows and one for many.  Down: h = x A_e^T, R values a row, summed in 32 bits; up: h B_e^T and the sum with base.
// Few rows: bound by launches and trips to memory.  The summed dimension is shared by the waves of a workgroup and by several workgroups, whose partial sums
// the second launch adds up; operands go from memory into the registers that multiply them.  Many rows: bound by reading x and base and writing y.
// h is not rounded to 16 bits on its way into the second product: it goes in as a sum of two (16-bit results) or, in bf16 with 32-bit results, three
// 16-bit numbers, 2^-16 (bf16), 2^-22 (f16) and 2^-24 of it off; the rank is short beside base and y, so the extra instructions are few.
#include "op_matmul_kernel.h"

#include <algorithm>

namespace sc {
namespace {

struct AdapterArgs {
    MatmulArgs g;                            // the groups: M, E, offsets
    const uint8_t* x;
    const int32_t* index;
    const uint8_t* a;
    const uint8_t* b;
    const float* scale;
    const void* base;
    void* y;
    float* h;                                // few rows: [splits][width / 4][M] of four ranks; many: the second product's operand (see adapters_down_wide_kernel)
    float* backs;                            // many rows, f16: [M], what takes a row's scaling back
    int32_t* place;                          // [rows]: place in the groups of a row that they name; anything for others
    int N, R, width, rows, kbytes, splits, pairs, up;        // pairs: 32 columns of y each, of a wave; up: workgroups that multiply
    int64_t x_row, a_row, a_adapter, b_row, b_adapter;       // bytes
    int64_t base_row, y_row;                 // elements
};

constexpr int kDownWaves = 8, kUpWaves = 4;
// ... of the second launch with many rows, and columns of a wave
constexpr int kWideWaves = 4, kWideColumns = 64;

// 16 RT WR rows a workgroup, RN tiles of 16 of R (more ranks are several workgroups'); WR waves along the rows times KW that share the summed
// dimension, a slab each in turn, the next one's operands on their way while one is multiplied.
template <int XT, int RN, int RT, int WR, int KW> __global__ __launch_bounds__(WR * KW * 64) void adapters_down_kernel(AdapterArgs p)
{
    constexpr int BT = 16 * RT * WR, W = WR * KW;
    __shared__ __align__(16) v4f part[W * RT * RN * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int parts = p.width / (RN * 16), tile = blockIdx.x / (p.splits * parts), at = blockIdx.x - tile * p.splits * parts, split = at / parts;
    const int r0 = (at - split * parts) * RN * 16;
    GroupTiles<BT> groups(p.g);
    if (tile >= groups.total) return;
    int e, first, m0, hi;
    groups.find(p.g, tile, e, first, m0, hi);
    m0 += (tile - first) * BT;
    const int rows = min(BT, hi - m0), wr = wave % WR, kw = wave / WR;
    const uint8_t* weights = p.a + e * p.a_adapter;
    const uint8_t* xrow[RT];
    uint32_t arow[RN];
#pragma unroll
    for (int j = 0; j < RT; ++j) {
        int t = m0 + min((wr * RT + j) * 16 + c, rows - 1);
        if (p.index) t = p.index[t];
        // (an index outside x: any row that can be read; its result is dropped)
        xrow[j] = ((uint32_t)t < (uint32_t)p.rows ? p.x + t * p.x_row : weights) + q * 16;
    }
#pragma unroll
    for (int i = 0; i < RN; ++i) arow[i] = (uint32_t)(min(r0 + i * 16 + c, p.R - 1) * p.a_row) + q * 16;
    const int slabs = (p.kbytes + kSlab - 1) / kSlab, each = (slabs + p.splits - 1) / p.splits, end = min(slabs, (split + 1) * each);
    v4f acc[RT][RN] = {};
    struct Operands { v4i x[RT][2], w[RN][2]; };
    auto load = [&](int s, Operands& o) {
        const int at0 = s * kSlab;
        if (at0 + kSlab <= p.kbytes) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < RT; ++j) o.x[j][h] = *reinterpret_cast<const v4i*>(xrow[j] + at0 + 64 * h);
#pragma unroll
                for (int i = 0; i < RN; ++i) o.w[i][h] = *reinterpret_cast<const v4i*>(weights + arow[i] + at0 + 64 * h);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // (what lies behind the end of a row is read from its last sixteen bytes and dropped)
                const int have = p.kbytes - at0 - 64 * h - q * 16, at = min(at0 + 64 * h, ((p.kbytes - 1) & ~15) - q * 16);
#pragma unroll
                for (int j = 0; j < RT; ++j) o.x[j][h] = first_bytes(*reinterpret_cast<const v4i*>(xrow[j] + at), have);
#pragma unroll
                for (int i = 0; i < RN; ++i) o.w[i][h] = first_bytes(*reinterpret_cast<const v4i*>(weights + (int)arow[i] + at), have);
            }
        }
    };
    auto multiply_all = [&](const Operands& o) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RN; ++i)
#pragma unroll
                for (int j = 0; j < RT; ++j) acc[j][i] = product16<XT>(o.w[i][h], o.x[j][h], acc[j][i]);
    };
    int s = split * each + kw;
    if (wr * RT * 16 < rows && s < end) {
        Operands one, two;
        load(s, one);
        for (;;) {
            if (s + KW < end) load(s + KW, two);
            multiply_all(one);
            if ((s += KW) >= end) break;
            if (s + KW < end) load(s + KW, one);
            multiply_all(two);
            if ((s += KW) >= end) break;
        }
    }
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int i = 0; i < RN; ++i) part[((kw * WR + wr) * RT * RN + j * RN + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    for (int v = threadIdx.x; v < WR * RT * RN * 64; v += W * 64) {
        v4f sum = part[v];
#pragma unroll
        for (int k = 1; k < KW; ++k) sum += part[k * WR * RT * RN * 64 + v];
        const int i = (v >> 6) % RN, row = (v >> 6) / RN * 16 + (v & 15);
        // (so that the second launch can tell the rows that no group names)
        if (p.index && p.place && at == 0 && row < rows && i == 0 && (v & 48) == 0) {
            const int t = p.index[m0 + row];
            if ((uint32_t)t < (uint32_t)p.rows) p.place[t] = m0 + row;
        }
        if (row < rows) reinterpret_cast<v4f*>(p.h)[((size_t)split * (p.width / 4) + r0 / 4 + i * 4 + ((v & 63) >> 4)) * p.g.M + m0 + row] = sum;
    }
}

// f as the sum of TERMS 16-bit numbers, the largest first.  (A bf16 of what lies above the largest one of them is that one, and the rest the next term's: rounded to
// an infinity it would leave another one, and their sum is a NaN.)
template <int XT, int TERMS, int N, class V> __device__ __forceinline__ void split_terms(const float* f, V (&out)[TERMS])
{
    float rest[N];
#pragma unroll
    for (int i = 0; i < N; ++i) rest[i] = f[i];
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            constexpr float kMost = 0x1.fep+127f;
            const bool finite = fabsf(rest[i]) < INFINITY;
            out[t][i] = (Elem<XT>)(XT == SC_ELEM_BF16 && t == 0 && finite ? __builtin_amdgcn_fmed3f(rest[i], -kMost, kMost) : rest[i]);
            rest[i] = finite ? rest[i] - (float)out[t][i] : 0.0f;
        }
}

// f16: a row's h, N of its values in each of the four lanes of it, is scaled by a power of two so that its largest value lies below 2^14, where no term
// leaves the type's range; returns what takes it back.
template <int XT, int N> __device__ __forceinline__ float row_scale(float* f)
{
    if constexpr (XT != SC_ELEM_F16) return 1.0f;
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(f[i]) < INFINITY ? fabsf(f[i]) : 0.0f);
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    const int exponent = max(__builtin_amdgcn_frexp_expf(most), -100);
    const float up = __builtin_amdgcn_ldexpf(1.0f, 14 - exponent);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] *= up;
    return __builtin_amdgcn_ldexpf(1.0f, exponent - 14);
}

template <int XT, int YT> constexpr int kTerms = YT == SC_ELEM_F32 && XT == SC_ELEM_BF16 ? 3 : 2;

// Many rows: sixteen a wave, W waves, all of R in RN tiles of 16.  Both operands are copied straight into LDS, 128 bytes of every row at a time, the
// next ST - 1 of these slabs under way (as in the tile of the products, whose layout in LDS this is).  What bounds it is how long a workgroup takes for a slab,
// for its way to LDS and the reads of it: so KS groups of W waves take every KS-th slab each, all in step, and the first adds the sums of the others to its own
// in their order (8192 x 4096 of rank 64: one group of four waves 20.0 us, two 16.6; 2048 rows: four waves 19.3, twice four 15.6, twice two 13.8, four times
// two 12.6).  h goes to the workspace as the second launch reads it: eight ranks of a term of
// all rows, then the next eight, so that the lanes of an operand, which are rows, read what lies in a row.
template <int XT, int YT, int RN, int W, int KS, int ST> __global__ __launch_bounds__(W * KS * 64) void adapters_down_wide_kernel(AdapterArgs p)
{
    constexpr int BT = 16 * W, XI = 2, AI = RN * 2 / W, COPIES = XI + AI, kStage = (BT + RN * 16) * kSlab, TERMS = kTerms<XT, YT>;
    static_assert(RN * 2 % W == 0, "copies");
    static_assert((KS - 1) * W * RN * 1024 <= ST * KS * kStage, "the groups' sums");
    __shared__ __align__(16) uint8_t lds[ST * KS * kStage];
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int kg = KS > 1 ? all / W : 0, wave = KS > 1 ? all % W : all;
    GroupTiles<BT> groups(p.g);
    // (neighbouring tiles on one die: few adapters' weights at a time in its second-level cache)
    const int total = groups.total;
    if ((int)blockIdx.x >= total) return;
    const int xcd = blockIdx.x & 7, tile = __builtin_amdgcn_readfirstlane(xcd * (total >> 3) + min(xcd, total & 7) + ((int)blockIdx.x >> 3));
    int e, first, m0, hi;
    groups.find(p.g, tile, e, first, m0, hi);
    m0 += (tile - first) * BT;
    const int rows = min(BT, hi - m0);
    // Copies: eight rows each, lane i brings sixteen bytes (i & 7) ^ key of row i >> 3.
    const uint8_t* weights = p.a + e * p.a_adapter;
    const uint8_t* src[COPIES];
    const int chunk = (lane & 7) ^ token_key(wave * 8 + (lane >> 3)), last = (p.kbytes - 1) >> 4;        // (copies of a wave are sixteen rows apart or 32: one key)
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        const int r = (i * W + wave) * 8 + (lane >> 3), m = m0 + min(r, rows - 1), t = p.index ? p.index[m] : m;
        const bool there = (uint32_t)t < (uint32_t)p.rows;
        // (an index outside x: any row that can be read; its result is dropped)
        src[i] = there ? p.x + t * p.x_row : weights;
        if (p.index && p.place && kg == 0 && there && r < rows && (lane & 7) == 0) p.place[t] = m;      // (for the rows that no group names: see rest_rows)
    }
#pragma unroll
    for (int i = 0; i < AI; ++i) src[XI + i] = weights + min((i * W + wave) * 8 + (lane >> 3), p.R - 1) * p.a_row;
    const int slabs = (p.kbytes + kSlab - 1) / kSlab, turns = (slabs + KS - 1) / KS, mine = (slabs - kg + KS - 1) / KS;     // of all groups; slabs of this one
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    auto stage = [&](int turn, int buf) {
        const int at = min((turn * KS + kg) * (kSlab / 16) + chunk, last) * 16;      // (what lies behind the end of a row is read from its last sixteen bytes and dropped)
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const uint32_t to = lds0 + (buf * KS + kg) * kStage + (i < XI ? 0 : BT * kSlab) + ((i < XI ? i : i - XI) * W + wave) * 1024;
            to_lds_ptr<16>(src[i] + at, to);
        }
    };
    v4f acc[RN] = {};
    const int key = lane_key(c);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (from here on only copies are counted)
    for (int s = 0; s < min(ST - 1, mine); ++s) stage(s, s);
    int buf = 0, next = ST - 1;
    auto slab = [&](int turn, auto cut) {    // cut: the last bytes of the rows, fewer than a slab
        constexpr bool CUT = decltype(cut)::value;
        const uint8_t* X = lds + (buf * KS + kg) * kStage;
        const int have = p.kbytes - (turn * KS + kg) * kSlab - q * 32;               // bytes of the row from this lane's on
        v4i x[2], w[2][RN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = *reinterpret_cast<const v4i*>(X + (wave * 16 + c) * kSlab + (((2 * q + h) ^ key) << 4));
#pragma unroll
            for (int i = 0; i < RN; ++i) w[h][i] = *reinterpret_cast<const v4i*>(X + (BT + i * 16 + c) * kSlab + (((2 * q + h) ^ key) << 4));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (CUT) x[h] = first_bytes(x[h], have - 16 * h);
#pragma unroll
            for (int i = 0; i < RN; ++i) acc[i] = product16<XT>(CUT ? first_bytes(w[h][i], have - 16 * h) : w[h][i], x[h], acc[i]);
        }
    };
    auto advance = [&] {
        buf = buf + 1 == ST ? 0 : buf + 1;
        next = next + 1 == ST ? 0 : next + 1;
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    const bool cut = p.kbytes % kSlab && (slabs - 1) % KS == kg;                     // (this group's last slab is the rows' last one, and short)
    int it = 0;
    for (; it + ST - 1 < mine; ++it) {
        staged<(ST - 2) * COPIES>();
        stage(it + ST - 1, next);
        slab(it, no);
        advance();
    }
    for (; it < turns; ++it) {               // (every group comes to every barrier)
        staged<0>();
        if (it < mine - cut) slab(it, no);
        else if (it < mine) slab(it, yes);
        advance();
    }
    if constexpr (KS > 1) {
        v4f* sums = reinterpret_cast<v4f*>(lds) + wave * RN * 64 + lane;
        __syncthreads();
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < RN; ++i) sums[((kg - 1) * W * RN + i) * 64] = acc[i];
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int i = 0; i < RN; ++i) acc[i] += sums[(k * W * RN + i) * 64];
    }
    // This lane's row (c) and four ranks of each sixteen: half of the sixteen bytes of a term of eight ranks.
    float f[RN][4];
#pragma unroll
    for (int i = 0; i < RN; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) f[i][v] = i * 16 + q * 4 + v < p.R ? acc[i][v] : 0.0f;
    const float back = row_scale<XT, RN * 4>(&f[0][0]);
    const int row = wave * 16 + c;
    if (row >= rows) return;
    const size_t m = m0 + row, M = p.g.M;
    if (XT == SC_ELEM_F16 && q == 0) p.backs[m] = back;
    uint8_t* z = reinterpret_cast<uint8_t*>(p.h);
#pragma unroll
    for (int i = 0; i < RN; ++i) {
        typedef Elem<XT> vec __attribute__((ext_vector_type(4)));
        vec term[TERMS];
        split_terms<XT, TERMS, 4>(f[i], term);
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
            __builtin_memcpy(z + ((size_t)((i / 2 * TERMS + t) * 4 + i % 2 * 2 + (q >> 1)) * M + m) * 16 + (q & 1) * 8, &term[t], 8);
    }
}

// Rows that no group names keep base: kRest of them a workgroup.  A row is named if the place that the first launch has noted for it holds it; what
// the workspace held before at a row that is not is some number, whose place is outside the groups or holds another row.
constexpr int kRest = 16;
template <int YT> __device__ __forceinline__ void rest_rows(const AdapterArgs& p, int block, int threads)
{
    const int lane = threadIdx.x & 63, t0 = block * kRest, t = min(t0 + (lane & (kRest - 1)), p.rows - 1);
    int lo = 0, hi = 0;
    if (p.g.M) lo = min(max(p.g.offsets[0], 0), p.g.M), hi = min(max(p.g.offsets[p.g.E], 0), p.g.M);
    bool named = lo <= t && t < hi;
    if (p.index && p.g.M) {
        const int at = p.place[t];
        named = lo <= at && at < hi && p.index[at] == t;
    }
    uint64_t rest = __ballot(!named && lane < kRest && t0 + lane < p.rows);
    for (; rest; rest &= rest - 1) {
        const int64_t row = t0 + __builtin_ctzll(rest);
        const Elem<YT>* from = static_cast<const Elem<YT>*>(p.base) + row * p.base_row;
        Elem<YT>* to = static_cast<Elem<YT>*>(p.y) + row * p.y_row;
        for (int col = threadIdx.x * 8; col < p.N; col += threads * 8) {
            float f[8];
            load_values<YT, 8>(from + col, p.N - col, f);
            store_values<YT, 8>(to + col, p.N - col, f);
        }
    }
}

// Few rows: sixteen a workgroup, its waves side by side along the columns; KT: R in steps of 32.  Two waves a SIMD up to 128 ranks, for which 32-bit results have up to four
// registers in scratch memory (768 rows of rank 128, f16: 28.7 us, with one wave a SIMD and none 32.7).
template <int XT, int YT, int KT> __global__ __launch_bounds__(kUpWaves * 64, KT < 8 ? 2 : 1) void adapters_up_kernel(AdapterArgs p)
{
    constexpr int TERMS = kTerms<XT, YT>;
    if ((int)blockIdx.x >= p.up) return rest_rows<YT>(p, blockIdx.x - p.up, kUpWaves * 64);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int blocks = (p.N + kUpWaves * 32 * p.pairs - 1) / (kUpWaves * 32 * p.pairs), tile = blockIdx.x / blocks, block = blockIdx.x - tile * blocks;
    GroupTiles<16> groups(p.g);
    if (tile >= groups.total) return;
    int e, first, m0, hi;
    groups.find(p.g, tile, e, first, m0, hi);
    m0 += (tile - first) * 16;
    const int rows = min(16, hi - m0), m = m0 + min(c, rows - 1), t = p.index ? p.index[m] : m;
    const bool there = (uint32_t)t < (uint32_t)p.rows, real = c < rows && there;
    const int64_t token = there ? t : 0;     // (base is read at a row that there is)
    const uint8_t* weights = p.b + e * p.b_adapter;
    // A lane's sixteen bytes of each step of its two rows (of two products a lane's sums are those of eight neighbouring columns: see the tile of the
    // products), from column n on.  What lies behind a row's end is read from its last sixteen bytes, and dropped.
    const int row[2] = {(c >> 2) * 8 + (c & 3), (c >> 2) * 8 + (c & 3) + 4};
    int at[KT];
#pragma unroll
    for (int k = 0; k < KT; ++k) at[k] = min(k * 64 + q * 16, (p.R * 2 - 1) & ~15);
    // (the step in which a row ends is one of the later half: what is kept of it; of the steps behind it, nothing)
    const int tail = (p.R * 2 - 1) >> 6;
    const v4i keep = first_bytes(v4i{-1, -1, -1, -1}, p.R * 2 - tail * 64 - q * 16);
    const Elem<YT>* from = static_cast<const Elem<YT>*>(p.base) + token * p.base_row + q * 8;
    Elem<YT>* to = static_cast<Elem<YT>*>(p.y) + token * p.y_row + q * 8;
    struct Pair { v4i w[2][KT]; float base[8]; };
    auto load = [&](int n, Pair& o) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < KT; ++k) o.w[i][k] = *reinterpret_cast<const v4i*>(weights + min(n + row[i], p.N - 1) * p.b_row + at[k]);
        load_values<YT, 8>(from + n, p.N - n - q * 8, o.base);
    };
    int n = (block * kUpWaves + wave) * 32 * p.pairs;
    const int end = min(n + 32 * p.pairs, p.N);
    if (n >= end) return;
    Pair one, two;
    load(n, one);                            // (before h, which is a trip of its own)
    v4i z[KT][TERMS];
    float f[KT][8] = {};
    const v4f* h = reinterpret_cast<const v4f*>(p.h) + m;
    const size_t M = p.g.M;
    const int four = KT > 1 || q * 8 < p.width ? q * 2 : 0;          // (16 ranks are half a step)
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            const size_t plane = (size_t)s * (p.width / 4) + k * 8 + four;
            const v4f lo = h[plane * M], high = h[(plane + 1) * M];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[k][i] += lo[i], f[k][4 + i] += high[i];
        }
    }
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k * 32 + q * 8 + i >= p.R) f[k][i] = 0.0f;
    const float scale = (p.scale ? p.scale[e] : 1.0f) * row_scale<XT, KT * 8>(&f[0][0]);
    typedef Elem<XT> terms __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        terms t[TERMS];
        split_terms<XT, TERMS, 8>(f[k], t);
        __builtin_memcpy(z[k], t, sizeof(t));
    }
    auto finish = [&](int n, Pair& o) {
        v4f acc[2] = {};
#pragma unroll
        for (int k = KT / 2; k < KT; ++k)
            if (k >= tail)
#pragma unroll
                for (int i = 0; i < 2; ++i) o.w[i][k] = k == tail ? o.w[i][k] & keep : v4i{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i] = product16<XT>(o.w[i][k], z[k][t], acc[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) o.base[i] = fmaf(scale, acc[i >> 2][i & 3], o.base[i]);
        if (real) store_values<YT, 8>(to + n, p.N - n - q * 8, o.base);
    };
    for (;;) {
        if (n + 32 < end) load(n + 32, two);
        finish(n, one);
        if ((n += 32) >= end) break;
        if (n + 32 < end) load(n + 32, one);
        finish(n, two);
        if ((n += 32) >= end) break;
    }
}

// Many rows: kChunk of a group a workgroup, whose waves have CW columns each and hold b of them in registers; sixteen rows at a time, the next ones' operands and base on their way.
// What bounds it is reading base and writing y, and the way there: a load takes a cycle of the address unit for each four lanes whose bytes lie in a
// row, and four if they do not, as in the order of the matrix operands (there sixteen lanes in a row are sixteen rows of b or y).  So the sums go through
// LDS, each wave's through its own, and are added to base and stored in rows, a workgroup's waves side by side: 64 columns a wave, whatever registers they take
// (us: rank 64, 8192 x 4096 39, with 32 columns 61, with 128 40; rank 128, 8192 x 2048 30, with 32 41; rank 256 50, with 32 63).
constexpr int kChunk = 128;
template <int XT, int YT, int KT> __global__ __launch_bounds__(kWideWaves * 64) void adapters_up_wide_kernel(AdapterArgs p)
{
    constexpr int TERMS = kTerms<XT, YT>, W = kWideWaves, CW = kWideColumns, NP = CW / 16;
    constexpr int V = kVec<YT>, LR = CW / V, PER = 64 / LR, U = 16 / PER, LINE = CW + 4;        // values and lanes of a row of y, rows at once, turns
    __shared__ __align__(16) float sums[W][16 * LINE];
    if ((int)blockIdx.x >= p.up) return rest_rows<YT>(p, blockIdx.x - p.up, W * 64);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int blocks = (p.N + W * CW - 1) / (W * CW), tile = blockIdx.x / blocks, block = blockIdx.x - tile * blocks, n0 = (block * W + wave) * CW;
    GroupTiles<kChunk> groups(p.g);
    if (tile >= groups.total || n0 >= p.N) return;
    int e, first, m0, hi;
    groups.find(p.g, tile, e, first, m0, hi);
    m0 += (tile - first) * kChunk;
    hi = min(hi, m0 + kChunk);

    // The rows of the chunk, two a lane.
    int tokens[kChunk / 64];
#pragma unroll
    for (int i = 0; i < kChunk / 64; ++i) {
        const int m = min(m0 + i * 64 + lane, hi - 1);
        tokens[i] = p.index ? p.index[m] : m;
    }
    // b of the wave's columns: of two products a lane's sums are those of eight neighbouring columns (see the tile of the products).  What lies behind a row's end
    // is read from its last sixteen bytes, and dropped.
    v4i w[NP][KT];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const uint8_t* row = p.b + e * p.b_adapter + min(n0 + (i >> 1) * 32 + (c >> 2) * 8 + (i & 1) * 4 + (c & 3), p.N - 1) * p.b_row;
#pragma unroll
        for (int k = 0; k < KT; ++k) w[i][k] = *reinterpret_cast<const v4i*>(row + min(k * 64 + q * 16, (p.R * 2 - 1) & ~15));
#pragma unroll
        for (int k = KT / 2; k < KT; ++k) w[i][k] = first_bytes(w[i][k], p.R * 2 - k * 64 - q * 16);         // (a row ends in one of the later half)
    }
    const float scale = p.scale ? p.scale[e] : 1.0f;
    const int col = n0 + lane % LR * V, have = p.N - col;
    struct Rows { v4i z[KT][TERMS], base[U]; float back; };
    const uint8_t* operands = reinterpret_cast<const uint8_t*>(p.h);
    // The row of y that turn u of the sixteen rows from i on (of the chunk) is for this lane; -1: none.
    auto row_of = [&](int i, int u) {
        const int r = i + lane / LR + u * PER, there = m0 + r < hi;
        const int t = __shfl(i < 64 ? tokens[0] : tokens[kChunk / 64 - 1], r & 63);
        return there && (uint32_t)t < (uint32_t)p.rows ? t : -1;
    };
    // `all`: all columns of the wave are there (then nothing branches between the loads, which would make each wait for all before it).
    auto load = [&](int i, Rows& o, auto all) {
        const size_t m = min(m0 + i + c, hi - 1), M = p.g.M;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int t = 0; t < TERMS; ++t) o.z[k][t] = *reinterpret_cast<const v4i*>(operands + ((size_t)((k * TERMS + t) * 4 + q) * M + m) * 16);
        if constexpr (XT == SC_ELEM_F16) o.back = p.backs[m];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Elem<YT>* from = static_cast<const Elem<YT>*>(p.base) + (int64_t)max(row_of(i, u), 0) * p.base_row + col;
            if constexpr (decltype(all)::value) o.base[u] = load_raw_once<YT>(from);
            else o.base[u] = have >= V ? load_raw<YT>(from) : load_raw_part<YT>(from, have);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    float* mine = sums[wave];
    auto finish = [&](int i, const Rows& o, auto all) {
        v4f acc[NP] = {};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
                for (int n = 0; n < NP; ++n) acc[n] = product16<XT>(w[n][k], o.z[k][t], acc[n]);
        const float by = XT == SC_ELEM_F16 ? scale * o.back : scale;
#pragma unroll
        for (int n = 0; n < NP; ++n) *reinterpret_cast<v4f*>(mine + c * LINE + (n >> 1) * 32 + q * 8 + (n & 1) * 4) = acc[n] * by;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = row_of(i, u);
            float f[V], g[V];
            to_floats<YT>(o.base[u], f);
            __builtin_memcpy(g, mine + (lane / LR + u * PER) * LINE + lane % LR * V, sizeof(g));
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] += g[v];
            Elem<YT>* to = static_cast<Elem<YT>*>(p.y) + (int64_t)max(t, 0) * p.y_row + col;
            if constexpr (decltype(all)::value) {
                if (t >= 0) store_once<YT, V>(to, f);
            } else if (t >= 0 && have > 0) {
                store_vec<YT, V>(to, f, have);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    const int n = hi - m0, last = (n - 1) & ~15;
    Rows one, two;
    if (n0 + CW <= p.N) {
        constexpr std::true_type all{};
        load(0, one, all);
        for (int i = 0;;) {
            load(min(i + 16, last), two, all);
            finish(i, one, all);
            if ((i += 16) >= n) break;
            load(min(i + 16, last), one, all);
            finish(i, two, all);
            if ((i += 16) >= n) break;
        }
    } else {
        constexpr std::false_type part{};
        for (int i = 0; i < n; i += 16) {
            load(i, one, part);
            finish(i, one, part);
        }
    }
}

constexpr int64_t kMaxRowBytes = (int64_t)1 << 22, kMaxAdapter = (int64_t)1 << 48;

sc_status_t check(const sc_adapters_t* d)
{
    if (!d) return SC_ERR_NULL;
    if (d->M < 0 || d->N <= 0 || d->K <= 0 || d->R <= 0 || d->R > 256 || d->E <= 0 || d->E > 4096 || d->rows < 0 || d->x_row < d->K || d->a_row < d->K || d->b_row < d->R ||
        d->base_row < 0 || d->y_row < d->N)
        return SC_ERR_SHAPE;
    if ((d->x_type != SC_ELEM_F16 && d->x_type != SC_ELEM_BF16) || (d->y_type != d->x_type && d->y_type != SC_ELEM_F32)) return SC_ERR_UNSUPPORTED;
    if (d->M > 1 << 30 || d->N > 1 << 30 || d->x_row >= kMaxRowBytes / 2 || d->a_row >= kMaxRowBytes / 2 || d->b_row >= kMaxRowBytes / 2 ||
        (d->E > 1 && (d->a_adapter >= kMaxAdapter || d->b_adapter >= kMaxAdapter)))
        return SC_ERR_RANGE;
    if (d->E > 1 && (d->a_adapter < (d->R - 1) * d->a_row + d->K || d->b_adapter < (d->N - 1) * d->b_row + d->R)) return SC_ERR_SHAPE;
    if (d->x_row % 8 || d->a_row % 8 || d->b_row % 8 || d->a_adapter % 8 || d->b_adapter % 8) return SC_ERR_UNSUPPORTED;
    return SC_OK;
}

// What a call runs: with many rows or few, workgroups that share the summed dimension and columns of a wave (few rows), workgroups.
//
// Many rows: from 1024 on, with ranks up to 32 from 2048, and 32 rows a group (us of both launches on the GPU, few and many, 4096 x 2048: rank 64, 768 rows
// 18 and 23, 1024 24 and 23, 2048 33 and 24; rank 32, 1536 rows 17 and 20, 2048 21 and 20; rank 256, 768 rows 53 and 53).
// In the first launch 32 rows a workgroup (`row_waves`) whose eight waves share the summed dimension, as long as every compute unit has one at most; then 64
// rows, as long as that holds for those, and beyond that the smaller workgroups again, two a compute unit, for ranks up to 64 (us: rank 64, 8192 rows 24 in the first,
// 17 in the second; rank 32, 16384 rows 44 in the second, 36 in the third; rank 128, 64 in the second and 74).
// Few rows: `splits` workgroups share the summed dimension, as many as keep the sum of both launches small: the first takes some 0.6 + 0.33 us a sixteen of
// ranks for each eight slabs, divided by them, the second 0.05 + 0.011 us a tile for 32 ranks of each part (measured, 4 to 1024 rows: the best of 1, 4, 8
// and 16 or within 4 % of it).
struct Shape { bool wide; int row_waves, shares, splits, pairs; int64_t down, up, rest; };

int rank_tiles(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : R <= 128 ? 8 : 16; }

Shape shape_of(const sc_adapters_t* d)
{
    Shape s{};
    const int rn = rank_tiles(d->R), groups = std::min(d->E, d->M);
    s.rest = ceil_div(d->rows, kRest);
    if (!d->M) return s;
    s.wide = d->M >= (rn <= 2 ? 2048 : 1024) && d->M >= 32 * (int64_t)groups;
    if (s.wide) {
        s.splits = s.pairs = 1;
        const bool fits = ceil_div(d->M, 32) + groups <= 256;
        s.row_waves = fits || (rn <= 4 && ceil_div(d->M, 64) + groups > 256) ? 2 : 4;
        s.shares = fits && rn < 16 ? 4 : 2;
        s.down = ceil_div(d->M, 16 * s.row_waves) + groups;
        s.up = (ceil_div(d->M, kChunk) + groups) * ceil_div(d->N, kWideWaves * kWideColumns);
        return s;
    }
    const int64_t tiles = ceil_div(d->M, 16) + groups, slabs = ceil_div(2 * (int64_t)d->K, kSlab);
    const double steps = (double)slabs / kDownWaves, first = (0.6 + 0.33 * std::min(rn, 4)) * steps, second = (0.05 + 0.011 * std::min<int64_t>(tiles, 32)) * std::max(rn / 2, 1);
    for (s.splits = 1; s.splits < 16 && s.splits * 2 <= steps && 2.0 * s.splits * s.splits * second <= first && tiles * s.splits * std::max(rn / 4, 1) <= 512; s.splits *= 2) {}
    s.down = tiles * s.splits * std::max(rn / 4, 1);
    s.pairs = (int)std::max<int64_t>(1, std::min<int64_t>(4, tiles * ceil_div(d->N, 32 * kUpWaves) / 256));
    s.up = tiles * ceil_div(d->N, 32 * kUpWaves * s.pairs);
    return s;
}

// h, what takes its rows' scaling back, the places
size_t h_bytes(const sc_adapters_t* d, const Shape& s)
{
    const size_t width = rank_tiles(d->R) * 16;
    if (!s.wide) return (size_t)s.splits * d->M * width * 4;
    const size_t terms = d->x_type == SC_ELEM_BF16 && d->y_type == SC_ELEM_F32 ? 3 : 2;
    return (std::max<size_t>(width, 32) * terms * 2 + 4) * d->M;
}
size_t workspace(const sc_adapters_t* d, const Shape& s) { return d->M ? h_bytes(d, s) + (size_t)d->rows * 4 : 0; }

template <int XT, int YT, int RN> sc_status_t launch_down(const AdapterArgs& a, const Shape& shape, hipStream_t s)
{
    const dim3 grid((unsigned)shape.down);
    constexpr int TILES = RN < 4 ? RN : 4, WIDE = RN < 2 ? 2 : RN;
    if (!shape.wide) {
        adapters_down_kernel<XT, TILES, 1, 1, 8><<<grid, kDownWaves * 64, 0, s>>>(a);
        return launched();
    }
    // (slabs in LDS: as many as leave it two workgroups, or one of eight waves, of 160 KiB)
    if (shape.row_waves == 4) adapters_down_wide_kernel<XT, YT, WIDE, 4, 2, WIDE < 8 ? 4 : WIDE < 16 ? 3 : 2><<<grid, 512, 0, s>>>(a);
    else if constexpr (WIDE < 16) {
        if (shape.shares == 4) adapters_down_wide_kernel<XT, YT, WIDE, 2, 4, WIDE < 8 ? 3 : 2><<<grid, 512, 0, s>>>(a);
        else if constexpr (WIDE < 8) adapters_down_wide_kernel<XT, YT, WIDE, 2, 2, WIDE < 4 ? 4 : 3><<<grid, 256, 0, s>>>(a);
    } else adapters_down_wide_kernel<XT, YT, WIDE, 2, 2, 2><<<grid, 256, 0, s>>>(a);
    return launched();
}

template <int XT, int YT, int RN> sc_status_t launch_up(const AdapterArgs& a, const Shape& shape, hipStream_t s)
{
    constexpr int KT = RN < 2 ? 1 : RN / 2;
    const dim3 grid((unsigned)(shape.up + shape.rest));
    if (!shape.wide) adapters_up_kernel<XT, YT, KT><<<grid, kUpWaves * 64, 0, s>>>(a);
    else adapters_up_wide_kernel<XT, YT, KT><<<grid, kWideWaves * 64, 0, s>>>(a);
    return launched();
}

template <int XT, int YT, int RN> sc_status_t launch_both(const AdapterArgs& a, const Shape& shape, hipStream_t s)
{
    const sc_status_t st = shape.down ? launch_down<XT, YT, RN>(a, shape, s) : SC_OK;
    return st == SC_OK ? launch_up<XT, YT, RN>(a, shape, s) : st;
}

template <int XT, int YT> sc_status_t launch_adapters(const AdapterArgs& a, const Shape& shape, hipStream_t s)
{
    switch (a.width) {
        case 16: return launch_both<XT, YT, 1>(a, shape, s);
        case 32: return launch_both<XT, YT, 2>(a, shape, s);
        case 64: return launch_both<XT, YT, 4>(a, shape, s);
        case 128: return launch_both<XT, YT, 8>(a, shape, s);
        default: return launch_both<XT, YT, 16>(a, shape, s);
    }
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_adapters_workspace_size(const sc_adapters_t* d, size_t* bytes)
{
    if (!bytes) return SC_ERR_NULL;
    const sc_status_t st = check(d);
    if (st == SC_OK) *bytes = workspace(d, shape_of(d));
    return st;
}

extern "C" sc_status_t sparse_conv_adapters_launch(const sc_adapters_t* d, sc_launch_t* launch)
{
    if (!launch) return SC_ERR_NULL;
    const sc_status_t st = check(d);
    if (st != SC_OK) return st;
    *launch = sc_launch_t{};
    if (d->M && d->rows) launch->form = shape_of(d).wide ? SC_FORM_ADAPTERS_MANY : SC_FORM_ADAPTERS_FEW;
    return SC_OK;
}

extern "C" sc_status_t sparse_conv_adapters(const sc_adapters_t* d, const void* x, const int32_t* index, const int32_t* offsets, const void* a, const void* b,
                                            const float* scale, const void* base, void* y, void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const sc_status_t st = check(d);
    if (st != SC_OK) return st;
    if (!index && d->rows < d->M) return SC_ERR_SHAPE;
    if (d->rows == 0) return SC_OK;
    if (!base || !y || (d->M && (!x || !offsets || !a || !b))) return SC_ERR_NULL;
    const int ye = elem_bytes(d->y_type);
    if (!aligned(x, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(index, 4) || !aligned(offsets, 4) || !aligned(scale, 4) || !aligned(base, ye) || !aligned(y, ye))
        return SC_ERR_UNSUPPORTED;
    const bool in_place = base == y && d->base_row == d->y_row;
    Shape shape = shape_of(d);
    if (in_place) shape.rest = 0;
    if (shape.up + shape.rest == 0) return SC_OK;
    if (shape.down * 512 >= (int64_t)1 << 32 || (shape.up + shape.rest) * 512 >= (int64_t)1 << 32) return SC_ERR_RANGE;        // (threads of a launch)
    if (d->M && (!workspace_dev || workspace_bytes < workspace(d, shape) || !aligned(workspace_dev, 16))) return SC_ERR_WORKSPACE;
    AdapterArgs p{};
    p.g.M = d->M; p.g.E = d->E; p.g.offsets = offsets;
    p.x = static_cast<const uint8_t*>(x); p.index = index; p.a = static_cast<const uint8_t*>(a); p.b = static_cast<const uint8_t*>(b);
    p.scale = scale; p.base = base; p.y = y; p.h = static_cast<float*>(workspace_dev);
    p.N = d->N; p.R = d->R; p.width = rank_tiles(d->R) * 16; p.rows = d->rows; p.kbytes = d->K * 2; p.splits = shape.splits; p.pairs = shape.pairs;
    p.up = (int)shape.up;
    p.backs = shape.wide ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + h_bytes(d, shape)) - d->M : nullptr;
    p.place = d->M && !in_place ? reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace_dev) + h_bytes(d, shape)) : nullptr;
    p.x_row = d->x_row * 2; p.a_row = d->a_row * 2; p.b_row = d->b_row * 2;
    p.a_adapter = d->E > 1 ? d->a_adapter * 2 : 0; p.b_adapter = d->E > 1 ? d->b_adapter * 2 : 0;
    p.base_row = d->base_row; p.y_row = d->y_row;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->y_type == SC_ELEM_F32;
    if (d->x_type == SC_ELEM_F16) return f32 ? launch_adapters<SC_ELEM_F16, SC_ELEM_F32>(p, shape, s) : launch_adapters<SC_ELEM_F16, SC_ELEM_F16>(p, shape, s);
    return f32 ? launch_adapters<SC_ELEM_BF16, SC_ELEM_F32>(p, shape, s) : launch_adapters<SC_ELEM_BF16, SC_ELEM_BF16>(p, shape, s);
}
