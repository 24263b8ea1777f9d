// The gradient of the stored weights, dvals[e] = sum over n of dZ(row of e, n) B(column of e, n): its kernels and the choice among them.
#include "gcoo_layer_values.hpp"
#include "gcoo_layer_device.hpp"
#include "gcoo_layer_long.hpp"
#include "gcoo_spdm_rows_kernel.hpp"

#include <algorithm>

namespace gcoo {

// ---- from the caches: entry by entry ----
//
// Sixteen lanes (a slot) are on a row of A: each holds P pieces of 16 bytes of the row of dZ in registers and takes the same pieces of the row of B of every entry, so that an
// entry costs P loads and 16 lanes x P pieces of multiply-adds.  Sixteen entries leave sixteen partial sums in every lane; they are added up by exchanging halves (the
// lanes that keep the upper eight sums give the lower eight to those that keep these, and so on), 45 instructions for sixteen entries instead of 128, after which lane i holds the sum of entry i.
// A wave has four rows beside each other, or all four slots on one row where it is long or rows are few.
//
// Bound: the vector caches, through which every entry takes its stretch of B.  The columns of B are cut into tiles of 256 P bytes that stay in an XCD's L2 (4 MB) for as many
// rows as A has columns; the sums of a tile go to `work` and values_join adds them in the order of the tiles (8000 x 8000, 0.5 %, N = 8000, bf16: 288 us, 8 of it the joining; 5.1 GB of rows of B, 18 TB/s).
// Long rows are cut into pieces for whole workgroups, which take them first (us, power-law rows, 16384 x 16384, of 53 entries, N = 300: bf16 694 124, fp32 287 124; even rows up to 0.3 us more).
constexpr int kLongPieces = 8;

template <int I>
__device__ __forceinline__ uint32_t slot_bcast(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + I, 0xf, 0xf, true); }      // row_newbcast:I

template <int CTRL>
__device__ __forceinline__ float lane_of(float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true)); }

// sums[i] of the slot's lanes -> the sum of all of sums[lane], in lane `lane` of the slot
template <int HALF, int CTRL>
__device__ __forceinline__ void exchange(float (&x)[16], int lane)
{
    const bool upper = lane & HALF;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
        const float keep = upper ? x[i + HALF] : x[i], give = upper ? x[i] : x[i + HALF];
        x[i] = keep + lane_of<CTRL>(give);
    }
}
__device__ __forceinline__ float slot_sums(float (&x)[16], int lane)
{
    exchange<8, 0x140>(x, lane);          // row_mirror: lane ^ 15
    exchange<4, 0x141>(x, lane);          // row_half_mirror: lane ^ 7
    exchange<2, 0x1b>(x, lane);           // quad_perm [3,2,1,0]: lane ^ 3
    exchange<1, 0xb1>(x, lane);           // quad_perm [1,0,3,2]: lane ^ 1
    return x[0];
}

template <typename T> struct Piece {
    static constexpr int kElements = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(kElements)));
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A lane's 16 bytes of a row of dZ, and their product with 16 bytes of a row of B, added to s.  bf16 stays in pairs: an instruction adds two exact products to a sum in fp32 and rounds once (checked against 64 bits, denormal
// numbers among them; the one for fp16 loses bits of those, where a multiply-add that takes one operand in fp16 does not).  With both operands widened, two instructions to an element, the
// vector instructions took 80 % of the time (8000 x 8000, 0.5 %, N = 8000: 292 us).
template <typename T> struct Held {
    float x[16 / sizeof(T)];
    __device__ __forceinline__ void set(const u32x4& w)
    {
        const typename Piece<T>::vec v = __builtin_bit_cast(typename Piece<T>::vec, w);
#pragma unroll
        for (int u = 0; u < Piece<T>::kElements; ++u) x[u] = widen((T)v[u]);
    }
    __device__ __forceinline__ float times(const u32x4& w, float s) const
    {
        const typename Piece<T>::vec v = __builtin_bit_cast(typename Piece<T>::vec, w);
#pragma unroll
        for (int u = 0; u < Piece<T>::kElements; ++u) s = __builtin_fmaf(x[u], widen((T)v[u]), s);
        return s;
    }
};
template <> struct Held<bf16_t> {
    typedef bf16_t pair __attribute__((ext_vector_type(2)));
    pair x[4];
    static __device__ __forceinline__ pair of(const u32x4& w, int u)
    {
        const uint32_t word = w[u];
        return __builtin_bit_cast(pair, word);
    }
    __device__ __forceinline__ void set(const u32x4& w)
    {
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = of(w, u);
    }
    __device__ __forceinline__ float times(const u32x4& w, float s) const
    {
#pragma unroll
        for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_fdot2_f32_bf16(x[u], of(w, u), s, false);
        return s;
    }
};

// B for a tile: by a buffer descriptor, or (ANY) by addresses in 64 bits, which serve a B of 4 GB and more and elements at odd places.
struct ValuesB {
    __amdgpu_buffer_rsrc_t rsrc;
    const char* base;
    uint64_t pitch;
};
constexpr uint32_t kNowhere = 0xfffff000u;         // beyond every descriptor, as is a lane's place in the tile added to it

// A lane's pieces: piece q begins at byte at[q] of the tile's rows, or is nothing (none[q]: its elements are 0); bits of `keep` say which of its bytes count.
template <typename T, int P>
struct Pieces {
    uint32_t at[P];
    bool none[P];
    u32x4 keep[P];
};

// Entries FROM .. FROM + CNT - 1 of the batch.
template <typename T, int P, bool PART, bool ANY, int FROM, int CNT, int I = 0>
__device__ __forceinline__ void values_load(uint32_t off, const Pieces<T, P>& pc, const ValuesB& B, u32x4 (&b)[CNT * P])
{
    if constexpr (I < CNT) {
        const uint32_t o = slot_bcast<FROM + I>(off);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if constexpr (ANY) {
                b[I * P + q] = 0u;
                if (o != kNowhere && !(PART && pc.none[q])) __builtin_memcpy(&b[I * P + q], B.base + (uint64_t)o * B.pitch + pc.at[q], 16);
            } else {
                b[I * P + q] = __builtin_amdgcn_raw_buffer_load_b128(B.rsrc, (int)(PART && pc.none[q] ? kNowhere : o + pc.at[q]), 0, 0);
            }
        }
        values_load<T, P, PART, ANY, FROM, CNT, I + 1>(off, pc, B, b);
    }
}

template <typename T, int P, bool PART, bool ANY, int FROM, int CNT>
__device__ __forceinline__ void values_batch(uint32_t off, const Pieces<T, P>& pc, const ValuesB& B, const Held<T> (&z)[P], float (&sums)[16])
{
    u32x4 b[CNT * P];
    values_load<T, P, PART, ANY, FROM, CNT>(off, pc, B, b);
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < P; ++q) {
            u32x4 w = b[i * P + q];
            if constexpr (PART) w &= pc.keep[q];
            s = z[q].times(w, s);
        }
        sums[FROM + i] = s;
    }
}

template <typename T, int P, bool PART, bool ANY>
struct ValuesTile {
    static constexpr int E = Piece<T>::kElements;
    const GradValuesArgs& a;
    float* out;
    Pieces<T, P> pc;
    ValuesB B;
    uint32_t kmax, pitch;
    int64_t j0;
    int lane;
    // `tile` of a launch whose first one is `tile0`
    __device__ __forceinline__ ValuesTile(const GradValuesArgs& args, int32_t tile0, int32_t tile, float* part) : a(args)
    {
        lane = threadIdx.x & 63;
        j0 = (int64_t)(tile0 + tile) * (16 * P * E);
        out = part ? part + (int64_t)tile * a.A.nnz : a.dvals;
        const int64_t N = a.N;
        // (a tile of fewer than E columns begins E in front of N: N is at least E)
        const int64_t first = j0 > N - E ? N - E : j0;
        const char* base = reinterpret_cast<const char*>(static_cast<const T*>(a.B) + first);
        const uint64_t bytes = ((uint64_t)(a.A.k - 1) * (uint64_t)a.ldb + (uint64_t)(N - first)) * sizeof(T);
        if constexpr (!ANY) B.rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)(uint32_t)bytes, 0x00027000);
        B.base = base;
        B.pitch = (uint64_t)a.ldb * sizeof(T);
        pitch = (uint32_t)B.pitch;
        kmax = (uint32_t)(a.A.k - 1);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int64_t want = j0 + (q * 16 + (lane & 15)) * E, begin = want > N - E ? N - E : want;
            pc.none[q] = PART && want >= N;
            pc.at[q] = (uint32_t)(begin - first) * (uint32_t)sizeof(T);
            if constexpr (PART) {
                // a piece that would reach beyond N lies in front of it instead: the elements that another lane has count 0
                const int skip = (int)(want - begin) * (int)sizeof(T);
#pragma unroll
                for (int w = 0; w < 4; ++w) pc.keep[q][w] = skip >= 4 * w + 4 ? 0u : (skip <= 4 * w ? ~0u : ~0u << (8 * (skip - 4 * w)));
            }
        }
    }
    __device__ __forceinline__ void row(int64_t r, Held<T> (&z)[P]) const
    {
        const char* src = reinterpret_cast<const char*>(static_cast<const T*>(a.dZ) + r * a.lddz + (j0 > a.N - E ? a.N - E : j0));
#pragma unroll
        for (int q = 0; q < P; ++q) {
            u32x4 w = 0u;
            if (!(PART && pc.none[q])) __builtin_memcpy(&w, src + pc.at[q], 16);
            if constexpr (PART) w &= pc.keep[q];
            z[q].set(w);
        }
    }
    __device__ __forceinline__ uint32_t offset(uint32_t e, uint32_t end) const
    {
        if (e >= end) return kNowhere;
        const uint32_t c = (uint32_t)a.A.cols[e], in = c < kmax ? c : kmax;
        return ANY ? in : in * pitch;
    }
    // The entries beg, beg + step, ... below end by sixteens, for each slot its own (every lane of the wave calls it).  (Unsigned: a step beyond the last of 2^31 entries stays a number.)
    __device__ __forceinline__ void entries(uint32_t beg, uint32_t end, uint32_t step, const Held<T> (&z)[P]) const
    {
        uint32_t e = beg + (uint32_t)(lane & 15);
        uint32_t next = offset(e, end);
        while (__any(e - (uint32_t)(lane & 15) < end)) {
            const uint32_t off = next;
            const uint32_t at = e;
            e += step;
            next = offset(e, end);
            // as many of the sixteen as the fullest slot of the wave has: a load past a row's end returns at once, but holds the address path as long as any other
            float sums[16];
            const int32_t left = (int32_t)(end - (at - (uint32_t)(lane & 15)));
            if constexpr (P == 1) {
                if (__any(left > 8)) values_batch<T, P, PART, ANY, 0, 16>(off, pc, B, z, sums);
                else if (__any(left > 4)) values_batch<T, P, PART, ANY, 0, 8>(off, pc, B, z, sums);
                else values_batch<T, P, PART, ANY, 0, 4>(off, pc, B, z, sums);
            } else if constexpr (P == 2) {
                if (__any(left > 4)) values_batch<T, P, PART, ANY, 0, 8>(off, pc, B, z, sums);
                else values_batch<T, P, PART, ANY, 0, 4>(off, pc, B, z, sums);
                if (__any(left > 12)) values_batch<T, P, PART, ANY, 8, 8>(off, pc, B, z, sums);
                else if (__any(left > 8)) values_batch<T, P, PART, ANY, 8, 4>(off, pc, B, z, sums);
            } else {
                values_batch<T, P, PART, ANY, 0, 4>(off, pc, B, z, sums);
                if (__any(left > 4)) values_batch<T, P, PART, ANY, 4, 4>(off, pc, B, z, sums);
                if (__any(left > 8)) values_batch<T, P, PART, ANY, 8, 4>(off, pc, B, z, sums);
                if (__any(left > 12)) values_batch<T, P, PART, ANY, 12, 4>(off, pc, B, z, sums);
            }
            const float s = slot_sums(sums, lane);
            if (at < end) out[at] = s;
        }
    }
    // A piece of a long row, by all slots of the workgroup.
    __device__ __forceinline__ void long_row(int32_t r, int32_t piece) const
    {
        const int32_t beg = a.A.start[r], end = a.A.start[r + 1];
        const int64_t n = end - beg;
        Held<T> z[P];
        row(r, z);
        entries((uint32_t)(beg + n * piece / kLongPieces) + 16 * (threadIdx.x >> 4), (uint32_t)(beg + n * (piece + 1) / kLongPieces), kValuesThreads, z);
    }
    // The row of this slot among rows r0 .. r0 + 3; `one`: r0 for all slots.
    __device__ __forceinline__ int64_t own(int64_t r0, bool one) const { return one ? r0 : r0 + (lane >> 4); }
    // Rows r0 .. r0 + 3, the slot's own of the entries [beg, end), but not long ones; `one`: row r0 by all slots.
    __device__ __forceinline__ void rows(int64_t r0, bool one, int32_t beg, int32_t end) const
    {
        const int slot = lane >> 4;
        const int64_t m = a.A.m, r = own(r0, one);
        if (end - beg > a.A.longs.long_row) end = beg;
        Held<T> z[P];
        if (!one) {
            // a row of more entries than the others of the wave together would have them wait: all slots take it
            const int32_t n = end - beg;
            int32_t all = n;
            all += __shfl_xor(all, 16, 64);
            all += __shfl_xor(all, 32, 64);
            const bool shared = n > 32 && n > 2 * (all - n);
            row(r < m ? r : m - 1, z);
            entries(beg, shared ? beg : end, 16, z);
            uint64_t todo = __ballot(shared && (lane & 15) == 0);
            while (todo) {                                       // wave-uniform
                const int s = (__ffsll((long long)todo) - 1) >> 4;
                todo &= todo - 1;
                const int32_t lb = __builtin_amdgcn_readlane(beg, 16 * s), le = __builtin_amdgcn_readlane(end, 16 * s);
                row(r0 + s, z);
                entries(lb + 16 * slot, le, 64, z);
            }
            return;
        }
        row(r < m ? r : m - 1, z);
        entries(beg + 16 * slot, end, 64, z);
    }
};

template <typename T, int P, bool ANY>
__global__ __launch_bounds__(kValuesThreads) void values_entries(GradValuesArgs a, float* part, int32_t tile0, int32_t tiles, int32_t row_wgs, int32_t one)
{
    // an XCD walks all rows of one tile before the next, eight tiles side by side; the tiles beyond the last whole eight are cut into eight slices of rows
    const int32_t block = (int32_t)blockIdx.x, xcd = block & 7, at = block >> 3, eights = tiles / 8;
    int32_t tile, wg, slice = 0;
    if (at < eights * row_wgs) {
        tile = at / row_wgs * 8 + xcd;
        wg = at - at / row_wgs * row_wgs;
    } else {
        const int32_t rest = (tiles - eights * 8) * row_wgs, x = at - eights * row_wgs;
        slice = (rest + 7) / 8;
        const int32_t i = xcd * slice + x;
        if (x >= slice || i >= rest) return;
        tile = eights * 8 + i / row_wgs;
        wg = i - i / row_wgs * row_wgs;
    }
    const int64_t wave = (int64_t)wg * (kValuesThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = one ? wave : 4 * wave;
    const int32_t turn = slice ? rows_slice_turn(tile - eights * 8, xcd, slice, row_wgs, wg) : wg;
    auto work = [&](const auto& t) {
        LongWalk<kLongPieces> walk(a.A.longs, a.A.start, a.A.m, turn, row_wgs);
        const int64_t r = t.own(r0, one);
        int32_t beg = 0, end = 0, row, piece;
        if (r < a.A.m) { beg = a.A.start[r]; end = a.A.start[r + 1]; }           // (on their way while the long rows are looked for)
        while (walk.next(&row, &piece)) t.long_row(row, piece);
        if (r0 < a.A.m) t.rows(r0, one, beg, end);
    };
    if ((int64_t)(tile0 + tile + 1) * (16 * P * Piece<T>::kElements) > a.N) work(ValuesTile<T, P, true, ANY>(a, tile0, tile, part));
    else work(ValuesTile<T, P, false, ANY>(a, tile0, tile, part));
}

// ---- few columns: a lane per entry ----
//
// Up to seven: sixteen lanes on a row of A, each on every sixteenth entry, the row of dZ in registers of all of them.
template <typename T, int MOST>
__global__ __launch_bounds__(kValuesThreads) void values_few(GradValuesArgs a)
{
    const int N = (int)a.N;
    const uint32_t kmax = (uint32_t)(a.A.k - 1);
    auto entries = [&](int64_t r, uint32_t beg, uint32_t end, uint32_t step) {
        const T* src = static_cast<const T*>(a.dZ) + r * a.lddz;
        float z[MOST];
#pragma unroll
        for (int j = 0; j < MOST; ++j) z[j] = j < N ? widen(src[j]) : 0.0f;
        for (uint32_t e = beg; e < end; e += step) {
            const uint32_t c = (uint32_t)a.A.cols[e];
            const T* b = static_cast<const T*>(a.B) + (int64_t)(c < kmax ? c : kmax) * a.ldb;
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < MOST; ++j)
                if (j < N) s = __builtin_fmaf(z[j], widen(b[j]), s);
            a.dvals[e] = s;
        }
    };
    int32_t row, piece;
    for (LongWalk<kLongPieces> walk(a.A.longs, a.A.start, a.A.m, (int32_t)blockIdx.x, (int32_t)gridDim.x); walk.next(&row, &piece);) {
        const int32_t beg = a.A.start[row], end = a.A.start[row + 1];
        const int64_t n = end - beg;
        entries(row, (uint32_t)(beg + n * piece / kLongPieces) + threadIdx.x, (uint32_t)(beg + n * (piece + 1) / kLongPieces), kValuesThreads);
    }
    const int64_t r = (int64_t)blockIdx.x * (kValuesThreads / 16) + (threadIdx.x >> 4);
    if (r >= a.A.m) return;
    const int32_t beg = a.A.start[r], end = a.A.start[r + 1];
    if (end - beg <= a.A.longs.long_row) entries(r, (uint32_t)beg + (threadIdx.x & 15), (uint32_t)end, 16);
}

// ---- by matrix instructions: whole tiles of dZ x B^T, of which the entries are taken ----
//
// For matrices that are not very sparse every product of a row of dZ and a row of B is computed, by matrix instructions, in tiles of TM rows of A x TN columns, and the stored entries
// are picked out of the tile's sums: 16-bit types reach sixteen times the rate of vector instructions so, and a row of B is fetched once per TM rows of A.  A tile without entries is not
// computed.  Both operands lie along N, 128 bytes of each row (a step) at a time: from memory to registers while the step before is multiplied, to LDS, and from
// there to the matrix instructions by 16 bytes per lane.  Where those bytes lie in a step is the same for both operands, so the instructions may take them in any order.
// 16 bytes of row r are at piece ^ (r / 2 mod 8) of its 128 in LDS: sixteen lanes that read one piece of sixteen rows, and sixteen that write two rows, meet all 64 banks once.
// For few tiles N is cut into parts, whose sums are joined afterwards.
// Bound: the matrix instructions (4001 x 3999, 5 %, N = 4003, bf16: 142 us with the starts, 0.84 of the rate of a large product, and 150 to 185 where pass follows pass; 8000 x 8000, 10 %, N = 8000: bf16 1.0 ms, fp32 8.1 ms, 127 of 153 TFLOP/s).
template <typename T> struct Mfma;
typedef float f32x16 __attribute__((ext_vector_type(16)));
template <> struct Mfma<bf16_t> {
    static __device__ __forceinline__ void step(const u32x4& a, const u32x4& b, f32x16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Piece<bf16_t>::vec, a), __builtin_bit_cast(Piece<bf16_t>::vec, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<f16_t> {
    static __device__ __forceinline__ void step(const u32x4& a, const u32x4& b, f32x16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Piece<f16_t>::vec, a), __builtin_bit_cast(Piece<f16_t>::vec, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<float> {
    static __device__ __forceinline__ void step(const u32x4& a, const u32x4& b, f32x16& c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    }
};

// starts[r][t] = the first entry of row r whose column is in tile t or behind it, t = 0 .. tiles; starts[r][0] = -1 where the columns of the row do not ascend.  A wave per row.
__global__ __launch_bounds__(kValuesThreads) void values_starts(RowsView A, int32_t tiles, int32_t tile_cols, int32_t* starts)
{
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * (kValuesThreads / 64) + (threadIdx.x >> 6);
    if (r >= A.m) return;
    int32_t* to = starts + r * (tiles + 1);
    const int32_t beg = A.start[r], end = A.start[r + 1];
    const uint32_t kmax = (uint32_t)(A.k - 1);
    auto tile_of = [&](int32_t e) {
        const uint32_t c = (uint32_t)A.cols[e];
        return (int32_t)((c < kmax ? c : kmax) / (uint32_t)tile_cols);
    };
    bool falls = false;
    for (int64_t e0 = beg; e0 < end; e0 += 64) {
        if (e0 + lane >= end) continue;
        const int32_t e = (int32_t)e0 + lane;
        const int32_t t = tile_of(e), before = e > beg ? tile_of(e - 1) : 0;
        falls |= before > t;
        for (int32_t x = before + 1; x <= t; ++x) to[x] = e;
        if (e == end - 1)
            for (int32_t x = t + 1; x <= tiles; ++x) to[x] = end;
    }
    if (end <= beg)
        for (int32_t x = 1 + lane; x <= tiles; x += 64) to[x] = beg;
    const bool any = __any(falls);
    if (lane == 0) to[0] = any ? -1 : beg;
}

// WM x WN waves, each MI x 2 tiles of 32 x 32.
template <typename T, int WM, int WN, int MI>
__global__ __launch_bounds__(64 * WM * WN, 2) void values_tiles(GradValuesArgs a, const int32_t* __restrict__ starts, float* out0, int32_t tiles_m, int32_t tiles_n, int32_t parts, int32_t part_steps)
{
    constexpr int TM = WM * MI * 32, TN = WN * 64, TH = 64 * WM * WN, E = Piece<T>::kElements, STEP = 8 * E, STAGE = (TM + TN) * 128, NA = TM * 8 / TH, NB = TN * 8 / TH;
    static_assert(TM * 8 % TH == 0 && TN * 8 % TH == 0 && TM <= TH && TH % 16 == 0, "pieces and rows of a thread");
    extern __shared__ __attribute__((aligned(16))) char smem[];               // two steps of both operands; then 64 rows of sums
    __shared__ int32_t from[TM], to[TM];
    const int t = (int)threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WN, wn = wave % WN;

    // An XCD has a stretch of the tiles, in groups of four rows of tiles, column by column: few rows of both operands at a time.
    const int32_t total = tiles_m * tiles_n * parts, per = (total + 7) / 8, item = (int32_t)(blockIdx.x & 7u) * per + (int32_t)(blockIdx.x >> 3);
    if (item >= total || (int32_t)(blockIdx.x >> 3) >= per) return;           // the whole workgroup
    const int32_t part = item / (tiles_m * tiles_n), at = item - part * (tiles_m * tiles_n), group = at / (4 * tiles_n), in = at - group * (4 * tiles_n);
    const int32_t high = tiles_m - 4 * group < 4 ? tiles_m - 4 * group : 4, tn = in / high, tm = 4 * group + in - tn * high;
    const int64_t m = a.A.m, k = a.A.k, N = a.N, r0 = (int64_t)tm * TM, c0 = (int64_t)tn * TN;

    // the entries of the tile, row by row
    int some = 0;
    if (t < TM) {
        int32_t f = 0, e = 0;
        if (r0 + t < m) {
            const int32_t* s = starts + (r0 + t) * (tiles_n + 1);
            if (s[0] < 0) { f = a.A.start[r0 + t]; e = a.A.start[r0 + t + 1]; }
            else { f = tn == 0 ? s[0] : s[tn]; e = s[tn + 1]; }
        }
        from[t] = f;
        to[t] = e;
        some = f < e;
    }
    if (!__syncthreads_or(some)) return;

    // this thread's pieces of a step: piece t % 8 of rows t / 8 + i TH / 8
    const char *pa[NA], *pb[NB];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int64_t r = r0 + t / 8 + i * (TH / 8);
        pa[i] = reinterpret_cast<const char*>(static_cast<const T*>(a.dZ) + (r < m ? r : m - 1) * a.lddz + (t & 7) * E);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int64_t c = c0 + t / 8 + i * (TH / 8);
        pb[i] = reinterpret_cast<const char*>(static_cast<const T*>(a.B) + (c < k ? c : k - 1) * a.ldb + (t & 7) * E);
    }
    const int64_t steps_all = (N + STEP - 1) / STEP, s0 = (int64_t)part * part_steps, s1 = s0 + part_steps < steps_all ? s0 + part_steps : steps_all;
    u32x4 va[NA], vb[NB];
    auto fetch = [&](int64_t s) {
        const int64_t n = N - s * STEP;
        if (n >= STEP) {
#pragma unroll
            for (int i = 0; i < NA; ++i) __builtin_memcpy(&va[i], pa[i] + s * 128, 16);
#pragma unroll
            for (int i = 0; i < NB; ++i) __builtin_memcpy(&vb[i], pb[i] + s * 128, 16);
        } else {
            // the last step: what is behind column N is 0 in both operands
            const int own = (int)n - (t & 7) * E;
            auto piece = [&](const char* p) {
                typename Piece<T>::vec x;
#pragma unroll
                for (int u = 0; u < E; ++u) x[u] = u < own ? reinterpret_cast<const T*>(p + s * 128)[u] : (T)0.0f;
                return __builtin_bit_cast(u32x4, x);
            };
#pragma unroll
            for (int i = 0; i < NA; ++i) va[i] = piece(pa[i]);
#pragma unroll
            for (int i = 0; i < NB; ++i) vb[i] = piece(pb[i]);
        }
    };
    // (TH / 8 is a multiple of 16 or 32: the swizzle of a thread's rows is the same for all of them)
    const int put_at = t / 8 * 128 + (((t & 7) ^ (t >> 4 & 7)) * 16);
    auto put = [&](char* stage) {
#pragma unroll
        for (int i = 0; i < NA; ++i) *reinterpret_cast<u32x4*>(stage + put_at + i * (TH / 8) * 128) = va[i];
#pragma unroll
        for (int i = 0; i < NB; ++i) *reinterpret_cast<u32x4*>(stage + TM * 128 + put_at + i * (TH / 8) * 128) = vb[i];
    };

    f32x16 acc[MI][2];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = 0.0f;
    const int l32 = lane & 31, half = lane >> 5, swizzle = l32 >> 1 & 7;
    const char *ga = smem + (wm * MI * 32 + l32) * 128, *gb = smem + (TM + wn * 64 + l32) * 128;
    fetch(s0);
    put(smem);
    __syncthreads();
    for (int64_t s = s0; s < s1; ++s) {
        const int stage = (int)((s - s0) & 1) * STAGE;
        if (s + 1 < s1) fetch(s + 1);
        u32x4 fa[2][MI], fb[2][2];
        auto read = [&](int q, u32x4 (&xa)[MI], u32x4 (&xb)[2]) {
            const int piece = stage + (((2 * q + half) ^ swizzle) * 16);
#pragma unroll
            for (int j = 0; j < 2; ++j) xb[j] = *reinterpret_cast<const u32x4*>(gb + j * 32 * 128 + piece);
#pragma unroll
            for (int i = 0; i < MI; ++i) xa[i] = *reinterpret_cast<const u32x4*>(ga + i * 32 * 128 + piece);
        };
        read(0, fa[0], fb[0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q < 3) read(q + 1, fa[(q + 1) & 1], fb[(q + 1) & 1]);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) Mfma<T>::step(fa[q & 1][i], fb[q & 1][j], acc[i][j]);
            // the next step to LDS: in front of the last quarter where a step is short (us, there and behind it: bf16, 4000 x 4000, N = 4000: 161 167, 2000 x 2000: 62 66; fp32: 1062 1030, 288 274)
            if (q == (sizeof(T) == 2 ? 2 : 3) && s + 1 < s1) put(smem + (STAGE - stage));
        }
        __syncthreads();
    }

    // 64 rows of sums at a time through LDS; TH / 64 threads take the entries of a row
    float* sums = reinterpret_cast<float*>(smem);
    float* out = out0 + (int64_t)part * a.A.nnz;
    const uint32_t kmax = (uint32_t)(k - 1);
    constexpr int LANES = TH / 64;
#pragma unroll
    for (int q = 0; q < TM / 64; ++q) {
        if (wm == q / (MI / 2)) {
            constexpr int PER = MI / 2;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int x = 0; x < 16; ++x)
                        sums[(i * 32 + 8 * (x / 4) + 4 * half + x % 4) * TN + wn * 64 + j * 32 + l32] = acc[(q % PER) * 2 + i][j][x];
        }
        __syncthreads();
        const int r = t / LANES;
        const uint32_t end = (uint32_t)to[q * 64 + r];
#pragma unroll 4
        for (uint32_t e = (uint32_t)(from[q * 64 + r] + t % LANES); e < end; e += LANES) {
            const uint32_t c = (uint32_t)a.A.cols[e], col = (c < kmax ? c : kmax) - (uint32_t)c0;
            if (col < (uint32_t)TN) out[e] = sums[r * TN + (int)col];
        }
        __syncthreads();
    }
}

// ---- dvals[e] = the sums of the tiles or parts, in their order; MORE: behind what it holds ----
template <bool MORE>
__global__ __launch_bounds__(kValuesThreads) void values_join(const float* __restrict__ part, float* __restrict__ dvals, int64_t nnz, int32_t parts)
{
    const int64_t e = (int64_t)blockIdx.x * kValuesThreads + threadIdx.x;
    if (e >= nnz) return;
    float s = part[e];
    if (MORE) s += dvals[e];
#pragma unroll 8
    for (int32_t i = 1; i < parts; ++i) s += part[(int64_t)i * nnz + e];
    dvals[e] = s;
}
static hipError_t launch_join(const float* part, float* dvals, int64_t nnz, int32_t parts, bool more, hipStream_t s)
{
    const auto kernel = more ? values_join<true> : values_join<false>;
    kernel<<<dim3((unsigned)((nnz + kValuesThreads - 1) / kValuesThreads)), dim3(kValuesThreads), 0, s>>>(part, dvals, nnz, parts);
    return hipGetLastError();
}

// ---- launches ----

template <typename T, int P>
static hipError_t launch_entries(const GradValuesArgs& a, const ValuesPlan& plan, float* part, hipStream_t s)
{
    constexpr int64_t waves = kValuesThreads / 64;
    const int64_t rows = plan.one ? waves : 4 * waves, row_wgs = (a.A.m + rows - 1) / rows;
    const auto kernel = plan.any ? values_entries<T, P, true> : values_entries<T, P, false>;
    for (int32_t tile0 = 0; tile0 < plan.parts; tile0 += plan.group) {
        const int64_t tiles = plan.parts - tile0 < plan.group ? plan.parts - tile0 : plan.group, rest = tiles % 8 * row_wgs, grid = tiles / 8 * 8 * row_wgs + (rest + 7) / 8 * 8;
        if (too_wide(grid, kValuesThreads)) return hipErrorInvalidConfiguration;
        kernel<<<dim3((unsigned)grid), dim3(kValuesThreads), 0, s>>>(a, plan.parts > 1 ? part : nullptr, tile0, (int32_t)tiles, (int32_t)row_wgs, plan.one ? 1 : 0);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && plan.parts > 1) e = launch_join(part, a.dvals, a.A.nnz, (int32_t)tiles, tile0 > 0, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t launch_few(const GradValuesArgs& a, hipStream_t s)
{
    constexpr int64_t rows = kValuesThreads / 16;
    if (too_wide((a.A.m + rows - 1) / rows, kValuesThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)((a.A.m + rows - 1) / rows)), threads(kValuesThreads);
    if (a.N <= 1) values_few<T, 1><<<grid, threads, 0, s>>>(a);
    else if (a.N <= 4) values_few<T, 4><<<grid, threads, 0, s>>>(a);
    else values_few<T, 8><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int WM, int WN, int MI>
static hipError_t launch_tiles(const GradValuesArgs& a, const ValuesPlan& plan, int32_t* starts, float* part, hipStream_t s)
{
    constexpr int TM = WM * MI * 32, TN = WN * 64, lds = 2 * (TM + TN) * 128;
    static_assert(64 * TN * 4 <= lds && TN == values_tile_cols(MI == 4), "the sums of 64 rows");
    static LdsLimit limit;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(&values_tiles<T, WM, WN, MI>), lds);
    if (e != hipSuccess) return e;
    const int64_t tiles_m = (a.A.m + TM - 1) / TM, tiles_n = (a.A.k + TN - 1) / TN, total = tiles_m * tiles_n * plan.parts;
    if (too_wide(total + 7, 64 * WM * WN) || too_wide((a.A.m + kValuesThreads / 64 - 1) / (kValuesThreads / 64), kValuesThreads)) return hipErrorInvalidConfiguration;
    const int64_t steps = (a.N * (int64_t)sizeof(T) + 127) / 128;
    values_starts<<<dim3((unsigned)((a.A.m + kValuesThreads / 64 - 1) / (kValuesThreads / 64))), dim3(kValuesThreads), 0, s>>>(a.A, (int32_t)tiles_n, TN, starts);
    values_tiles<T, WM, WN, MI><<<dim3((unsigned)((total + 7) / 8 * 8)), dim3(64 * WM * WN), lds, s>>>(a, starts, plan.parts > 1 ? part : a.dvals, (int32_t)tiles_m, (int32_t)tiles_n, plan.parts,
                                                                                   (int32_t)((steps + plan.parts - 1) / plan.parts));
    const hipError_t launched = hipGetLastError();
    return launched != hipSuccess || plan.parts == 1 ? launched : launch_join(part, a.dvals, a.A.nnz, plan.parts, false, s);
}

// Times of the two kernels, in microseconds, of which the shorter is taken.  Entries: what they take of B through the vector caches, both matrices from memory once.  Tiles: all products of
// m x k x N, then the entries one by one.  Against 126 products (256 to 8000 rows and columns, N = 64 to 8000, 0.5 to 20 % stored, bf16 and fp32) the one so chosen takes 1.5 % longer than the faster of
// the two on average (bf16, us, entries and tiles: 8000 x 8000, N = 8000, 1 %: 545 977, 5 %: 2226 1011; 4000 x 4000, N = 4000, 2 %: 131 147, 5 %: 296 148; 2000 x 2000, N = 512, 5 %: 16 20, 10 %: 24 21;
// fp32: 8000 x 8000, N = 8000, 5 %: 4411 8088, 20 %: 16597 8141; 2000 x 2000, N = 4000, 10 %: 246 272).
// `slower`: what rows at odd places (1.76) or inside 128-byte lines, of which a tile takes one more than it has bytes for, make of the former.
static double entries_time(double nnz, double rows, double bytes, double slower) { return 5.0 + nnz * bytes * slower / 22e6 + rows * bytes / 5e6; }
static double tiles_time(double m, double k, double nnz, double N, int type)
{
    return (type == GCOO_F32 ? 15.0 : 12.0) + 2.0 * m * k * N / (type == GCOO_F32 ? 0.122e9 : 0.9e9) + nnz * 5e-6;
}

ValuesPlan values_plan(int64_t m, int64_t k, int64_t nnz, int64_t N, int type, const void* B, int64_t ldb)
{
    const int64_t size = (int64_t)type_bytes(type), bytes = N * size;
    ValuesPlan p{kValuesFew, 1, 1, 1, false, false, 0, 0};
    // (from eight columns on a slot of 16 lanes takes 16 bytes a lane and nothing beside them; us, a lane per entry and so: bf16, 8000 x 8000, 5 %, N = 8: 40 38, 16: 71 39, 32: 213 38; 0.5 %, N = 32: 43 10; fp32, 5 %,
    // N = 4: 27 35, 8: 42 35, 16: 110 35; power-law rows, 16384 x 16384, of 53, bf16, N = 8: 41 36, 32: 136 35)
    if (N < 8) return p;
    // (buffer loads at multiples of 4 bytes only)
    p.any = (uint64_t)k * (uint64_t)ldb * (uint64_t)size > kRowsMaxBytes || reinterpret_cast<uintptr_t>(B) % 4 != 0 || ldb * size % 4 != 0 || bytes % 4 != 0;
    // Rows of 2-byte elements at odd places, and rows inside lines where there are several tiles: as they are, or copied first (us, as they are and so: 20000 x 20000, rows of 40: bf16, N = 700: 145 99, fp32, N = 300: 124 87;
    // 12000 x 12000, rows of 100, bf16, N = 1000: 168 143; 6000 x 6000, rows of 40, N = 1000: 37 as they are, 38 so).
    const bool odd = odd_rows(B, ldb, type), lines = ldb * size % 128 == 0 && reinterpret_cast<uintptr_t>(B) % 128 == 0;
    const double inside = lines || bytes <= 1024 ? 1.0 : 1.0 + (double)k / 40000.0, slower = odd && inside < 1.76 ? 1.76 : inside;
    const double as_is = entries_time((double)nnz, (double)(m + k), (double)bytes, slower);
    const double copied = entries_time((double)nnz, (double)(m + k), (double)bytes, 1.0) + 2.0 + 2.0 * (double)size * (double)k * (double)N / 4.5e6;
    const bool copies = copied < (odd ? 1.0 : 0.95) * as_is;
    if (tiles_time((double)m, (double)k, (double)nnz, (double)N, type) < (copies ? copied : as_is)) {
        // tiles of 256 x 256 where they fill the compute units, else of 128 x 128 and as many parts of N as fill them twice, of four steps and more
        p.kernel = kValuesTiles;
        p.pieces = type != GCOO_F32 && ((m + 255) / 256) * ((k + 255) / 256) >= 160 ? 4 : 2;
        const int64_t edge = values_tile_cols(p.pieces == 4), tiles_n = (k + edge - 1) / edge, tiles = ((m + edge - 1) / edge) * tiles_n, steps = (bytes + 127) / 128;
        const int64_t wanted = p.pieces == 4 ? 1 : (512 + tiles - 1) / tiles, most = (steps + 3) / 4, parts = wanted < most ? wanted : most, each = (steps + parts - 1) / parts;
        p.parts = p.group = (int32_t)((steps + each - 1) / each);          // none of them empty
        p.starts = m * (tiles_n + 1);
        return p;
    }
    // The widest tile of B of which an XCD's L2 keeps all rows (us, 1, 2 and 4 pieces: bf16, 0.5 %: 2000 x 2000, N = 4000: 24.6 22.6 22.1; 4000 x 4000, N = 4000: 53.0 48.6 47.4; 8000 x 8000, N = 8000:
    // 319 297 379; 14000 x 14000, N = 2000: 287 342 398; fp32: 4000 x 4000, N = 4000: 82 70 76; 8000 x 8000, N = 8000: 581 563 778), and one tile where N allows it.
    p.kernel = kValuesEntries;
    if (copies) {
        p.ldw = (N + 63) / 64 * 64;
        p.any = (uint64_t)k * (uint64_t)p.ldw * (uint64_t)size > kRowsMaxBytes || bytes % 4 != 0;
    }
    if (bytes <= 1024) p.pieces = bytes <= 256 ? 1 : (bytes <= 512 ? 2 : 4);
    else p.pieces = k <= 3500 ? 4 : (k <= 10000 ? 2 : 1);
    p.parts = (int32_t)((bytes + 256 * p.pieces - 1) / (256 * p.pieces));
    // As many tiles to a launch as leave kValuesSums of their sums, but eight at the least, one to an XCD; all of about the same number.  (A launch more costs the end of one, where workgroups of long rows are alone: us, fp32,
    // one launch, 1 GB and 256 MB of sums: 14000 x 14000, 16.7 million entries, N = 2653: 7638 7758 8132; 5.9 million, N = 8000: 8663 8716 8934; 12000 x 12000, 4 %, N = 8000: 8034 8188 8370.  The sums would grow with
    // N: 3 GB for the first two.)
    const int64_t most = std::max<int64_t>(kValuesSums / nnz / 8 * 8, 8), launches = (p.parts + most - 1) / most;
    p.group = launches > 1 ? (int32_t)(((p.parts + launches - 1) / launches + 7) / 8 * 8) : p.parts;
    p.one = m * p.parts < 4096 && nnz >= 12 * m;
    return p;
}

hipError_t launch_grad_values(const GradValuesArgs& args, const ValuesPlan& plan, int32_t* starts, float* part, void* copy, hipStream_t s)
{
    GradValuesArgs a = args;
    hipError_t e = hipSuccess;
    if (plan.ldw > 0) {
        const int64_t halves = (int64_t)type_bytes(a.type) / 2;
        e = launch_realign(a.B, a.ldb * halves, copy, plan.ldw * halves, a.A.k, a.N * halves, s);
        if (e != hipSuccess) return e;
        a.B = copy;
        a.ldb = plan.ldw;
    }
    return with_type(a.type, [&](auto t) {
        typedef decltype(t) T;
        if (plan.kernel == kValuesFew) return launch_few<T>(a, s);
        if (plan.kernel == kValuesTiles) {
            if constexpr (sizeof(T) == 2)
                if (plan.pieces == 4) return launch_tiles<T, 2, 4, 4>(a, plan, starts, part, s);
            return launch_tiles<T, 2, 2, 2>(a, plan, starts, part, s);
        }
        return plan.pieces == 1 ? launch_entries<T, 1>(a, plan, part, s) : (plan.pieces == 2 ? launch_entries<T, 2>(a, plan, part, s) : launch_entries<T, 4>(a, plan, part, s));
    });
}

}  // namespace gcoo
