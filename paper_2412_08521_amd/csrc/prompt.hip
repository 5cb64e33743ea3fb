// Attention of many queries: o_i = sum_t p_t v_t / sum_t p_t with p_t = exp(scale q_i.k_t - m), lse_i = m + ln sum_t p_t, over the
// live rows t <= i + m - n that query i of n sees of m rows.  One pass with a running reference m and sum.
//
// prompt_kernel  bfloat16.  A block takes a tile of query rows of one kv-head, the group's q-heads of a token side by side (row
//                token * group + head), and walks the rows of keys and values in stages through LDS that all its waves read:
//                  S^T = K Q^T    32x32x16 products; a lane holds one query's column, 16 of a tile's 32 rows
//                  O^T = V^T P^T  S^T's registers are the right operand as they are; the left one is read transposed
// prompt_f32     the same with 32-bit rows and products, plain
// prompt_join    a tile whose rows several blocks share: their outputs, weighted by their references and sums
//
// What bounds it.  A 32x32x16 product takes a SIMD 8 passes (32 clocks) and needs, at 32 query rows a wave, 1 KiB of LDS; a tile
// of 32 x 32 weights takes three and a half instructions a weight (multiply-add, exponential, sum, half a conversion) beside D/4 products.  64
// query rows a wave halve the reads of LDS, and with products of one step beside the weights of another the matrix units
// are what is left: 32 q-heads on 8, D = 128, a prompt of 32768 tokens takes 7.1 to 7.4 ms from card to card (1.24 to 1.19 PFLOP/s; a
// plain product of matrices reaches 1.37 at its best size).  With one step at a time and one register tile it took 22.0 ms, with three
// in flight 7.8 ms, with fewer instructions for addresses and edges 7.2 ms.  The same without the weights' instructions would run at
// 1.47 PFLOP/s, without the loads of stages at 1.36; tiles drawn from a counter at run time gained 1.5 % at that size and lost 1 %
// at 1024 tokens, so a block has one tile.  (All of these with the wait that the compiler places in a stage, see below.)  At D = 64
// a tile of 32 x 32 weights is 256 clocks of products and, counted, some 400 of weights' instructions (an exponential as four).
//
// The weights are rounded to bfloat16 for the second product (relative 2^-8 each, as the values and the output are); their sum is
// of the 32-bit ones.  Beside the output's own rounding (0.0017 of it, root mean square) that leaves 0.0019 to 0.0024; whole weights
// would be three products for one, as few columns over pages have them, which memory bounds.
#include <cmath>

#include "ems_common.h"
#include "ems_kernels.h"
#include "ems_rows.h"
#include "ems_stream.h"

namespace ems {

namespace {

constexpr int kNoRow = -1;

// A sequence: its queries, its rows, and where they begin.
struct Seq { int n, m, q_first, k_first; };

template <bool kPaged>
__device__ __forceinline__ Seq sequence(const PromptArgs& a, int b)
{
    if constexpr (kPaged) {
        const long long most = (long long)a.max_pages * a.page_size;
        const int n = a.new_len ? min(max(a.new_len[b], 0), a.q_rows) : a.q_rows;
        return {n, (int)min((long long)max(a.lens[b], 0), most), b * a.q_rows, 0};
    }
    if (!a.q_start) return {a.q_rows, a.k_rows, b * a.q_rows, 0};
    const int q0 = min(max(a.q_start[b], 0), a.q_rows), q1 = min(max(a.q_start[b + 1], q0), a.q_rows);
    const int k0 = min(max(a.k_start[b], 0), a.k_rows), k1 = min(max(a.k_start[b + 1], k0), a.k_rows);
    return {q1 - q0, k1 - k0, q0, k0};
}

// Which sequence and tile of kRowsOf query rows is the j-th of a kv-head; b = -1: there are not as many.  Tiles with the most rows to
// see come first: blocks begin in this order, and the last ones are then short.
struct Place { int b, tile, n_tiles; Seq seq; };
__device__ __forceinline__ int tiles_of_rows(long long rows, int rows_of) { return (int)((rows + rows_of - 1) / rows_of); }

template <bool kPaged>
__device__ __forceinline__ Place find_tile(const PromptArgs& a, int j, int rows_of)
{
    const int lane = threadIdx.x % kWave;
    if (kPaged ? a.batch == 1 || (a.batch > kWave && !a.new_len) : !a.q_start) {         // tiles of every sequence alike
        const int b = j % a.batch;
        const Seq s = sequence<kPaged>(a, b);
        const int n = tiles_of_rows((long long)s.n * a.group, rows_of), t = n - 1 - j / a.batch;
        return {t >= 0 ? b : -1, t, n, s};
    }
    const auto from_lane = [](const Seq& s, int b) {
        return Seq{__builtin_amdgcn_readlane(s.n, b), __builtin_amdgcn_readlane(s.m, b), __builtin_amdgcn_readlane(s.q_first, b),
                   __builtin_amdgcn_readlane(s.k_first, b)};
    };
    const auto total = [](int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); };
    if (a.batch <= kWave) {
        // tile t of a sequence has level base + t: the tiles' worth of rows that its queries see, about
        const Seq s = lane < a.batch ? sequence<kPaged>(a, lane) : Seq{0, 0, 0, 0};
        const int n = tiles_of_rows((long long)s.n * a.group, rows_of);
        const int base = s.m > s.n ? (int)min((long long)(s.m - s.n) * a.group / rows_of, 1ll << 29) : 0;
        const auto from = [&](int level) { return total(min(max(base + n - level, 0), n)); };         // tiles of that level and above
        int lo = 0, hi = n ? base + n : 0;                     // from(lo) > j >= from(hi)
        for (int x = 1; x < kWave; x *= 2) hi = max(hi, __shfl_xor(hi, x));
        hi = scalar(hi);
        int above = 0;                                         // from(hi)
        if (from(0) <= j) return {-1, 0, 0, s};
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1, x = from(mid);
            if (x > j) lo = mid;
            else { hi = mid; above = x; }
        }
        const bool has = n > 0 && base <= lo && lo < base + n;
        const unsigned long long those = __ballot(has);
        const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(those >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)those, 0));
        const int b = __builtin_ctzll(__ballot(has && before == j - above));
        return {b, lo - __builtin_amdgcn_readlane(base, b), __builtin_amdgcn_readlane(n, b), from_lane(s, b)};
    }
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {              // many sequences: in their order
        const Seq s = b0 + lane < a.batch ? sequence<kPaged>(a, b0 + lane) : Seq{0, 0, 0, 0};
        const int n = tiles_of_rows((long long)s.n * a.group, rows_of), sum = wave_scan(n);
        const unsigned long long past = __ballot(sum > j);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int n_at = __builtin_amdgcn_readlane(n, at);
            return {b0 + at, __builtin_amdgcn_readlane(sum, at) - 1 - j, n_at, from_lane(s, at)};
        }
        j -= __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0, 0, Seq{0, 0, 0, 0}};
}

// Bytes of LDS that a stage of keys (or values) takes, and where its pieces of 16 bytes are: a row's pieces change places by
// the row's number, so that what lanes read together lies in different banks.
template <typename T, int D> struct Stage {
    static constexpr int kRows = sizeof(T) == 2 ? 64 : 32;
    static constexpr int kRowBytes = D * (int)sizeof(T), kPieces = kRowBytes / 16;
    static constexpr int kBytes = kRows * kRowBytes;
    static constexpr int kDma = kBytes / 1024, kDmaRows = 1024 / kRowBytes;      // instructions, and rows of one
    // keys: a product's 32 lanes read a piece of 32 rows
    static __device__ __forceinline__ int key(int row) { return swz_key<T, D>(row); }
    // values: 16-bit ones are read transposed, 32 lanes four pieces of four rows; 32-bit ones a row's 32 elements
    static __device__ __forceinline__ int value(int row)
    {
        if constexpr (sizeof(T) == 4) return 0;
        return kPieces == 16 ? 4 * (row & 3) : 4 * ((row ^ (row >> 1)) & 1);
    }
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ s16x4_t read_transposed(unsigned lds)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(uintptr_t)lds);
}

// 16 bytes of a row; `wide`: the address is a multiple of 16 bytes
template <typename T>
__device__ __forceinline__ frag_t load_piece(const T* p, bool wide)
{
    if (wide) return *reinterpret_cast<const frag_t*>(p);
    struct Elems { T x[16 / sizeof(T)]; } e;
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e.x[i] = p[i];
    return __builtin_bit_cast(frag_t, e);
}

// Four elements of a row; `wide`: the row starts at a multiple of 16 bytes
template <typename T>
__device__ __forceinline__ void store4(T* p, float x0, float x1, float x2, float x3, bool wide)
{
    struct alignas(4 * sizeof(T)) Elems { T x[4]; } e{{(T)x0, (T)x1, (T)x2, (T)x3}};
    if (wide) *reinterpret_cast<Elems*>(p) = e;
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = e.x[i];
    }
}

// A condition that hardly ever holds: what copies registers need go to its side.
__device__ __forceinline__ bool rare(bool x) { return __builtin_expect_with_probability(x, 0, 0.9999); }

constexpr int kMinusInf = (int)0xff800000;

// Four bytes a lane from global memory to LDS; wait_vmem counts it.
__device__ __forceinline__ void dma4(const void* from, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(scalar((int)lds)) : "memory", "m0");
}

// What the wave has read from LDS is in its registers: DMA may write there.
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// From global memory to LDS, a piece of 16 bytes a lane, from the wave's address on; wait_vmem counts it.
__device__ __forceinline__ void dma16(const char* from, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(scalar((int)lds)) : "memory", "m0");
}

// The same for two or four instructions on neighbouring KiB of LDS, from `base` on by 32-bit offsets or from 64-bit addresses.  An
// instruction's own offset (0, 1024, ..) counts on both sides, so those that are passed are that much lower (kDmaBias higher).
constexpr unsigned kDmaBias = 3 * 1024;
template <int kN>
__device__ __forceinline__ void dma_group(const void* base, const unsigned (&off)[kN], unsigned lds)
{
    const char* b = static_cast<const char*>(base) - kDmaBias;
    if constexpr (kN == 4)
        asm volatile("s_mov_b32 m0, %5\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %4 offset:1024\n\t"
                     "global_load_lds_dwordx4 %2, %4 offset:2*1024\n\tglobal_load_lds_dwordx4 %3, %4 offset:3*1024"
                     ::"v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(b), "s"(lds) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %3\n\tglobal_load_lds_dwordx4 %0, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024"
                     ::"v"(off[0]), "v"(off[1]), "s"(b), "s"(lds) : "memory", "m0");
}
template <int kN>
__device__ __forceinline__ void dma_group(const char* const (&from)[kN], unsigned lds)
{
    if constexpr (kN == 4)
        asm volatile("s_mov_b32 m0, %4\n\tglobal_load_lds_dwordx4 %0, off\n\tglobal_load_lds_dwordx4 %1, off offset:1024\n\t"
                     "global_load_lds_dwordx4 %2, off offset:2*1024\n\tglobal_load_lds_dwordx4 %3, off offset:3*1024"
                     ::"v"(from[0]), "v"(from[1]), "v"(from[2]), "v"(from[3]), "s"(lds) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, off\n\tglobal_load_lds_dwordx4 %1, off offset:1024"
                     ::"v"(from[0]), "v"(from[1]), "s"(lds) : "memory", "m0");
}

}  // namespace

// 32-bit rows: a wave takes a tile of 32 query rows, a stage is 32 rows, and its products come one after the other (32x32x2, a value
// a lane).  The products bound it: 16 x the time of 16-bit ones, beside which the loads and weights do not show.
template <int D, bool kPaged>
__global__ __launch_bounds__(128, 2) void prompt_f32_kernel(PromptArgs a)
{
    typedef float T;
    using St = Stage<T, D>;
    constexpr int kW = 2, kKv = St::kRows;
    static_assert(kKv == 32, "a tile of rows");
    constexpr int kFrags = Tile<T, D>::kFrags, kOut = D / 32;
    constexpr int kRowsOf = 32 * kW;
    constexpr int kHold = 4;                                   // tiles whose rows are known
    __shared__ __align__(1024) char stage[2][2][St::kBytes];
    __shared__ int row_of[kPaged ? kHold : 1][kKv];
    __shared__ unsigned live_of[kPaged ? kHold : 1];

    const int lane = threadIdx.x % kWave, wave = scalar((int)threadIdx.x / kWave);
    const int col = lane % 32, half = lane / 32;
    const int head = blockIdx.x % a.kv_heads, split = blockIdx.y;
    const Place place = find_tile<kPaged>(a, blockIdx.x / a.kv_heads, kRowsOf);
    if (place.b < 0) return;
    const int b = scalar(place.b), tile = scalar(place.tile);
    const Seq seq{scalar(place.seq.n), scalar(place.seq.m), scalar(place.seq.q_first), scalar(place.seq.k_first)};
    const int n_rows = seq.n * a.group;                        // (the host holds it to 31 bits)
    const int r0 = tile * kRowsOf + 32 * wave;
    const int row = min(r0 + col, n_rows - 1);
    const int token = row / a.group, q_head = head * a.group + row - token * a.group;
    const int lim = min(token + 1 + seq.m - seq.n, seq.m);     // rows that the lane's query sees (none: <= 0)
    const int lim_min = __builtin_amdgcn_readlane(lim, 0), lim_max = __builtin_amdgcn_readlane(lim, 31);
    const int last_token = min(tile * kRowsOf + kRowsOf - 1, n_rows - 1) / a.group;
    const int rows_end = min(max(last_token + 1 + seq.m - seq.n, 0), seq.m);
    const int n_stages = (rows_end + kKv - 1) / kKv;
    const int lo = (int)((long long)n_stages * split / a.splits), hi = (int)((long long)n_stages * (split + 1) / a.splits);

    frag_t qf[kFrags];
    {
        const T* q = reinterpret_cast<const T*>(a.q) + q_head * a.q_sh + (a.q_start ? (seq.q_first + token) * a.q_sn : b * a.q_sb + token * a.q_sn);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) qf[f] = load_piece(q + (2 * f + half) * 4, a.q_wide);
    }

    // ---- rows of a stage
    struct Look { int entry, row, mask; };
    const auto page_of = [&](int t) { return (int)(__umulhi(2u * (unsigned)t, a.page_magic) >> a.page_shift); };
    const auto table_trip = [&](int it) -> int {
        const int t = it * kKv + lane;
        return it >= lo && lane < kKv && t < rows_end ? a.page_table[(size_t)b * a.max_pages + page_of(t)] : kNoRow;
    };
    const auto row_trip = [&](int it, int entry, int& mask) -> int {
        const int t = it * kKv + lane;
        mask = 0;
        if (entry < 0 || entry >= a.num_pages) return kNoRow;
        const int r = (entry * a.kv_heads + head - page_of(t)) * a.page_size + t;
        if (a.pos_pages) mask = a.pos_pages[r];
        return r;
    };
    const auto settle = [&](int it, int r, int mask) {
        if (mask < 0) r = kNoRow;
        const unsigned live = (unsigned)__ballot(r != kNoRow); // (of lanes 0 .. 31: the others have no row)
        const int spare = live ? __builtin_amdgcn_readlane(r, __builtin_ctz(live)) : 0;
        if (lane < kKv) row_of[it % kHold][lane] = r != kNoRow ? r : spare;
        if (lane == 0) live_of[it % kHold] = live;
    };

    const unsigned lds = lds_address(&stage[0][0][0]);
    const auto load_stage = [&](int it, int buf) {
#pragma unroll
        for (int i = 0; i < (St::kDma + kW - 1) / kW; ++i) {
            const int n = i * kW + wave;                       // instruction: kDmaRows rows from n * kDmaRows on
            if (St::kDma % kW != 0 && n >= St::kDma) break;
            const int r = n * St::kDmaRows + lane / St::kPieces, p = lane % St::kPieces;
            const char *k, *v;
            if constexpr (kPaged) {
                const size_t at = (size_t)(unsigned)row_of[it % kHold][r] * St::kRowBytes;
                k = reinterpret_cast<const char*>(a.k) + at;
                v = reinterpret_cast<const char*>(a.v) + at;
            } else {
                const long long t = seq.k_first + min(it * kKv + r, seq.m - 1);
                const long long kb = a.q_start ? 0 : b * a.k_sb, vb = a.q_start ? 0 : b * a.v_sb;
                k = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.k) + kb + head * a.k_sh + t * a.k_sn);
                v = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.v) + vb + head * a.v_sh + t * a.v_sn);
            }
            k += 16 * (p ^ St::key(r));
            v += 16 * (p ^ St::value(r));
            if (kPaged || a.kv_wide) {
                dma16(k, lds + (2 * buf) * St::kBytes + 1024 * n);
                dma16(v, lds + (2 * buf + 1) * St::kBytes + 1024 * n);
            } else {
                *reinterpret_cast<frag_t*>(&stage[buf][0][1024 * n + 16 * lane]) = load_piece(reinterpret_cast<const T*>(k), false);
                *reinterpret_cast<frag_t*>(&stage[buf][1][1024 * n + 16 * lane]) = load_piece(reinterpret_cast<const T*>(v), false);
            }
        }
    };

    f32x16_t o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i) o[i] = zero_acc();
    float m = -INFINITY, l = 0.f;                              // of the lane's query; l: this lane's rows only

    const unsigned k_base = lds + col * St::kRowBytes + 16 * (half ^ St::key(col));
    unsigned v_base[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i) {
        v_base[i] = lds + St::kBytes + 4 * half * St::kRowBytes + 4 * (32 * i + col);
    }
    const auto lds_frag = [](unsigned at) { return *(const __attribute__((address_space(3))) frag_t*)(uintptr_t)at; };
    const auto lds_float = [](unsigned at) { return *(const __attribute__((address_space(3))) float*)(uintptr_t)at; };

    const auto compute = [&](int it, int buf, auto masked, unsigned live, bool edge) {
        constexpr bool kMasked = decltype(masked)::value;
        const unsigned off = 2 * buf * St::kBytes;
        f32x16_t s = zero_acc();
#pragma unroll
        for (int f = 0; f < kFrags; ++f) mma<T>(s, lds_frag((k_base ^ (32 * f)) + off), qf[f]);
        unsigned seen = 0;
        if constexpr (kMasked) {
            const int left = lim - it * kKv;                   // rows of this stage that the query sees
            seen = ((left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1) & live) >> (4 * half);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (seen >> acc_row(r, 0)) & 1 ? s[r] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = halves_max(top) * a.scale_log2e;
        // the reference stays until a logit exceeds it by 8 powers of two: sums and outputs have the room
        if (__any(top > m + 8.f)) {
            const float m_new = fmaxf(m, top), ref = m_new > -INFINITY ? m_new : 0.f;
            const float shrink = exp2_fast(m - ref);
            l *= shrink;
#pragma unroll
            for (int i = 0; i < kOut; ++i) o[i] *= shrink;
            m = m_new;
        }
        const float ref = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = exp2_fast(__builtin_fmaf(s[r], a.scale_log2e, -ref));
            l += s[r];
        }
        const auto value_row = [&](int r, int i) { return lds_float(v_base[i] + off + acc_row(r, 0) * St::kRowBytes); };
        // Where some query does not see a row, the row's value counts 0 times: an infinity or NaN there must not.  Such a stage
        // (hardly ever there) adds values that are finite, and sees by a second product which queries see one that is not.
        bool odd = false;
        if constexpr (kMasked) if (edge) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int i = 0; i < kOut; ++i) odd |= !(fabsf(value_row(r, i)) < INFINITY);
            odd = __any(odd);
        }
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            f32x16_t count = zero_acc();
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = value_row(r, i);
                if (kMasked && odd) {
                    const bool fine = fabsf(x) < INFINITY;
                    count = __builtin_amdgcn_mfma_f32_32x32x2f32(fine ? 0.f : 1.f, (seen >> acc_row(r, 0)) & 1 ? 1.f : 0.f, count, 0, 0, 0);
                    x = fine ? x : 0.f;
                }
                o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[r], o[i], 0, 0, 0);
            }
            if (kMasked && odd)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] = count[r] > 0.f ? NAN : o[i][r];
        }
    };

    // Stages come last rows first.  One is in flight while one is worked on; rows of pages are looked up two further on, a stage a turn.
    int entry = kNoRow, far = kNoRow, far_mask = 0;
    if constexpr (kPaged) {
        if (wave == 0 && hi > lo) {
#pragma unroll
            for (int i = 1; i <= 2; ++i) {
                int mask;
                const int r = row_trip(hi - i, table_trip(hi - i), mask);
                settle(hi - i + kHold, r, mask);               // (hi - 2 may be -1)
            }
            far = row_trip(hi - 3, table_trip(hi - 3), far_mask);
            entry = table_trip(hi - 4);
        }
        __syncthreads();
    }
    if (hi > lo) load_stage(hi - 1 + (kPaged ? kHold : 0), 0);
    for (int it = hi - 1, buf = 0; it >= lo; --it, buf ^= 1) {
        wait_vmem_all_visible();
        __syncthreads();
        if (it > lo) load_stage(it - 1, buf ^ 1);
        unsigned live = ~0u;
        if constexpr (kPaged) {
            live = (unsigned)scalar((int)live_of[it % kHold]);
            if (wave == 0) {
                settle(it - 2 + kHold, far, far_mask);
                far = row_trip(it - 3, entry, far_mask);
                entry = table_trip(it - 4);
            }
        }
        if (r0 < n_rows && it * kKv < lim_max && live) {
            const bool edge = it * kKv + kKv > lim_min;
            if (edge || (kPaged && live != ~0u)) compute(it, buf, std::true_type{}, live, edge);
            else compute(it, buf, std::false_type{}, ~0u, false);
        }
    }

    // ---- the lane's query: columns 32 i + acc_row(r, half)
    l = halves_sum(l);
    if (r0 + col >= n_rows) return;
    const float ref = m > -INFINITY ? m : 0.f;
    const long long q_token = seq.q_first + token;
    if (a.splits > 1) {
        const long long at = (q_token * a.kv_heads * a.group + q_head) * a.splits + split;
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 32 * i + acc_row(r, half)) = f32x4_t{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
        if (half == 0) { a.part_ml[2 * at] = m; a.part_ml[2 * at + 1] = l; }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;                // (NaN stays)
    T* out = reinterpret_cast<T*>(a.out) + q_head * a.o_sh + (a.q_start ? q_token * a.o_sn : b * a.o_sb + token * a.o_sn);
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) store4(out + 32 * i + acc_row(r, half), o[i][r] * inv, o[i][r + 1] * inv, o[i][r + 2] * inv, o[i][r + 3] * inv, a.o_wide);
    if (a.lse && half == 0) a.lse[(a.q_start ? q_token : b * a.l_sb + token) + q_head * a.l_sh] = (ref + log2_fast(l)) * 0.6931471805599453f;
}

// 16-bit rows.  A wave takes kQ tiles of 32 query rows (64 where there are many: every row of keys and values that it reads from
// LDS goes into two products) and works on three steps of 32 rows at once, products of one beside the weights of another:
//     S(n) = K(n) Q^T,   P(n - 1) = exp2(S(n - 1) - m),   O += V(n - 2)^T P(n - 2)^T
// kSome: rows of the cache are masked (by their positions); their logits begin at -inf.
// kS: waves that share the rows of keys and values of one tile (then kW = 1).  Each walks a part of its own, 32 rows a stage, and
// meets the others at the end.
template <int D, bool kPaged, bool kSome, int kQ, int kW, int kS>
__global__ __launch_bounds__(64 * kW * kS, D == 128 && kQ == 2 ? 1 : 2) void prompt_kernel(PromptArgs a)
{
    typedef bf16_t T;
    using St = Stage<T, D>;
    constexpr int kKv = St::kRows, kRowsOfLoad = kS > 1 ? 32 : kKv, kLoadBytes = kRowsOfLoad * St::kRowBytes;
    static_assert(kS == 1 || (kW == 1 && kQ == 1), "one tile");
    constexpr int kFrags = Tile<T, D>::kFrags, kOut = D / 32;
    constexpr int kRowsOf = 32 * kQ * kW;
    constexpr int kBatch = 4, kHold = 2 * kBatch;              // stages whose rows are looked up together, and are known
    __shared__ __align__(1024) char rings[kS][5][kLoadBytes];              // two of keys, three of values
    __shared__ int rows_of[kS][kPaged ? kHold : 1][kKv];
    __shared__ unsigned long long lives_of[kS][kPaged ? kHold : 1];
    __shared__ int founds[kS][kPaged ? kBatch : 1][2][kWave];  // table elements and positions

    const int lane = threadIdx.x % kWave, number = scalar((int)threadIdx.x / kWave);
    const int wave = kS > 1 ? 0 : number, part = kS > 1 ? number : 0;
    auto& row_of = rows_of[part];
    auto& live_of = lives_of[part];
    auto& found = founds[part];
    char (&keys)[5][kLoadBytes] = rings[part];
    char* const vals = rings[part][2];
    const int col = lane % 32, half = lane / 32;
    const int split = blockIdx.y * kS + part, splits = a.splits * kS;
    const int head = blockIdx.x % a.kv_heads;
    const Place place = find_tile<kPaged>(a, blockIdx.x / a.kv_heads, kRowsOf);
    if (scalar(place.b) < 0) return;
    const int b = scalar(place.b), tile = scalar(place.tile);
    const Seq seq{scalar(place.seq.n), scalar(place.seq.m), scalar(place.seq.q_first), scalar(place.seq.k_first)};
    const int n_rows = seq.n * a.group;                        // (the host holds it to 31 bits)
    const int r0 = tile * kRowsOf + 32 * kQ * wave;
    // the query of a lane: its token and q-head
    struct Query { int token, head; };
    const auto query = [&](int c, int col) __attribute__((always_inline)) {
        const int row = min(r0 + 32 * c + col, n_rows - 1), token = row / a.group;
        return Query{token, head * a.group + row - token * a.group};
    };
    const auto sees = [&](int token) __attribute__((always_inline)) { return min(token + 1 + seq.m - seq.n, seq.m); };    // rows (none: <= 0)
    const int lim_min = scalar(sees(query(0, 0).token)), lim_max = scalar(sees(query(kQ - 1, 31).token));
    const int last_token = min(tile * kRowsOf + kRowsOf - 1, n_rows - 1) / a.group;
    const int rows_end = min(max(last_token + 1 + seq.m - seq.n, 0), seq.m);
    const int n_stages = (rows_end + kKv - 1) / kKv;
    const int lo = (int)((long long)n_stages * split / splits), hi = (int)((long long)n_stages * (split + 1) / splits);

    frag_t qf[kQ][kFrags];
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
        const Query at = query(c, col);
        const T* q = reinterpret_cast<const T*>(a.q) + at.head * a.q_sh + (a.q_start ? (seq.q_first + at.token) * a.q_sn : b * a.q_sb + at.token * a.q_sn);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) qf[c][f] = load_piece(q + (2 * f + half) * 8, a.q_wide);
    }

    // ---- rows of a stage, found four stages at a time: a batch's stages are the waves', one after the other.  The trips of the
    // batch below are made while one is worked on (the table; positions; then its rows are settled), from memory to LDS, so that
    // no register waits for them: the loads of the stages are in flight behind them.  (Not so where waves share a tile: there
    // the first step after a trip waits for it before it asks for the next rows, in one stage of four, in two with positions.)
    constexpr int kMine = kBatch / kW;
    static_assert(kBatch % kW == 0, "every wave has as many");
    const auto page_of = [&](int t) __attribute__((always_inline)) { return (int)(__umulhi(2u * (unsigned)t, a.page_magic) >> a.page_shift); };
    const auto look_up = [&](int batch, int trip) __attribute__((always_inline)) {
        if (batch < 0) return;
        const int lane = lane_here();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int n = wave * kMine + i, it = batch * kBatch + n, t = min(it * kKv + lane, a.max_pages * a.page_size - 1), page = page_of(t);
            if (trip == 0) {
                dma_to_lds<4>(a.page_table + (size_t)b * a.max_pages, 4u * (unsigned)page, lds_address(&found[n][0][0]));
                continue;
            }
            const int entry = found[n][0][lane];
            int r = kNoRow;
            if (it >= lo && it * kKv + lane < rows_end && entry >= 0 && entry < a.num_pages) r = (entry * a.kv_heads + head - page) * a.page_size + t;
            if (trip == 1) {
                if constexpr (kSome) dma4(a.pos_pages + max(r, 0), lds_address(&found[n][1][0]));
                continue;
            }
            if (kSome && found[n][1][lane] < 0) r = kNoRow;
            const unsigned long long live = __ballot(r != kNoRow);
            const int spare = live ? __builtin_amdgcn_readlane(r, __builtin_ctzll(live)) : 0;
            row_of[it % kHold][lane] = r != kNoRow ? r : spare;
            if (lane == 0) live_of[it % kHold] = live;
        }
    };

    const unsigned k_lds = lds_address(&keys[0][0]), v_lds = lds_address(vals);
    // A stage's rows go to LDS by kDma instructions, neighbouring ones of which are a wave's, in groups under one LDS address.
    constexpr int kDma = kLoadBytes / 1024, kLoads = kDma / kW, kGroup = kLoads < 4 ? kLoads : 4;
    static_assert(kDma % kW == 0 && kLoads % kGroup == 0 && (kGroup == 2 || kGroup == 4), "every wave has whole groups");
    const auto row_of_load = [&](int i, int lane) __attribute__((always_inline)) { return (wave * kLoads + i) * St::kDmaRows + lane / St::kPieces; };
    const auto key_piece = [&](int i, int lane) __attribute__((always_inline)) { return 16 * (lane % St::kPieces ^ St::key(row_of_load(i, lane))); };
    const auto value_piece = [&](int i, int lane) __attribute__((always_inline)) { return 16 * (lane % St::kPieces ^ St::value(row_of_load(i, lane))); };
    const char* k_first = nullptr;                             // the sequence's rows
    const char* v_first = nullptr;
    const char* k_next = nullptr;                              // those of the stage that is loaded next
    const char* v_next = nullptr;
    const long long k_step = a.k_sn * (long long)sizeof(T), v_step = a.v_sn * (long long)sizeof(T);       // bytes from row to row
    // from a stage's first row (the host holds strides to 24 bits); held, but where the registers do not suffice
    constexpr bool kHeld = D == 128 || kQ == 1;
    const auto offset_of = [&](auto values_, int i, int lane) __attribute__((always_inline)) {
        constexpr bool kValues = decltype(values_)::value;
        return (unsigned)row_of_load(i, lane) * (unsigned)(kValues ? v_step : k_step) + (kValues ? value_piece(i, lane) : key_piece(i, lane)) + kDmaBias - 1024 * (i % kGroup);
    };
    unsigned k_off[kLoads], v_off[kLoads];
    if constexpr (!kPaged) {
        k_first = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.k) + (a.q_start ? 0 : b * a.k_sb) + head * a.k_sh + seq.k_first * a.k_sn);
        v_first = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.v) + (a.q_start ? 0 : b * a.v_sb) + head * a.v_sh + seq.k_first * a.v_sn);
        k_next = k_first + (long long)(hi * kKv - kRowsOfLoad) * k_step;
        v_next = v_first + (long long)(hi * kKv - kRowsOfLoad) * v_step;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) { k_off[i] = offset_of(std::false_type{}, i, lane); v_off[i] = offset_of(std::true_type{}, i, lane); }
    }
    // kRowsOfLoad rows of one stage from row `first` on, keys or values, to LDS at `to`
    const auto load_rows = [&](auto values_, int first, unsigned to) __attribute__((always_inline)) {
        constexpr bool kValues = decltype(values_)::value;
        const int lane = lane_here();
        const auto piece = [&](int i) __attribute__((always_inline)) { return kValues ? value_piece(i, lane) : key_piece(i, lane); };
        const int it = first / kKv, mine = kLoads * wave;
        to = scalar((int)to) + 1024 * mine;
        typedef __attribute__((address_space(3))) frag_t* lds_frag_t;
        if constexpr (kPaged) {
            const char* rows = reinterpret_cast<const char*>(kValues ? a.v : a.k);
            if (live_of[it % kHold] == 0) {                    // nothing there: zeros, which count nothing
#pragma unroll
                for (int i = 0; i < kLoads; ++i) *(lds_frag_t)(uintptr_t)(to + 1024 * i + 16 * lane) = zero_frag();
                return;
            }
#pragma unroll
            for (int g = 0; g < kLoads; g += kGroup) {
                const char* from[kGroup];
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                    from[i] = rows + piece(g + i) - 1024 * i + (unsigned long long)(unsigned)row_of[it % kHold][first % kKv + row_of_load(g + i, lane)] * St::kRowBytes;
                dma_group<kGroup>(from, to + 1024 * g);
            }
            return;
        }
        const char* rows = kValues ? v_first : k_first;
        const long long step = kValues ? v_step : k_step;
        const char*& next = kValues ? v_next : k_next;
        if (!rare(!a.kv_wide || first + kRowsOfLoad > seq.m)) {
#pragma unroll
            for (int g = 0; g < kLoads; g += kGroup) {
                unsigned off[kGroup];
#pragma unroll
                for (int i = 0; i < kGroup; ++i) off[i] = !kHeld ? offset_of(values_, g + i, lane) : kValues ? v_off[g + i] : k_off[g + i];
                dma_group<kGroup>(next, off, to + 1024 * g);
            }
        } else if (a.kv_wide) {                                // rows past the last are read as the last
#pragma unroll
            for (int g = 0; g < kLoads; g += kGroup) {
                const char* from[kGroup];
#pragma unroll
                for (int i = 0; i < kGroup; ++i) {
                    const unsigned t = min(first + row_of_load(g + i, lane), seq.m - 1);
                    from[i] = rows + t * (unsigned long long)(unsigned)step + piece(g + i) - 1024 * i;
                }
                dma_group<kGroup>(from, to + 1024 * g);
            }
        } else {
#pragma unroll 4
            for (int i = 0; i < kLoads; ++i) {
                const long long t = min(first + row_of_load(i, lane), seq.m - 1);
                *(lds_frag_t)(uintptr_t)(to + 1024 * i + 16 * lane) = load_piece(reinterpret_cast<const T*>(rows + t * step + piece(i)), false);
            }
        }
        next -= kRowsOfLoad * step;
    };

    // ---- the wave's state
    f32x16_t o[kQ][kOut], s[2][kQ];                            // s: of the step whose products run, and of the one before
    frag_t p[2][kQ][2];                                        // weights, the same way
    frag_t kf[kFrags], vf[2][kOut];
    float m[kQ], l[kQ];                                        // of the lane's queries (m: NaN before the first); l: this lane's rows only
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
#pragma unroll
        for (int i = 0; i < kOut; ++i) o[c][i] = zero_acc();
#pragma unroll
        for (int r = 0; r < 16; ++r) s[1][c][r] = -INFINITY;
        p[1][c][0] = p[1][c][1] = zero_frag();
        m[c] = NAN; l[c] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < kOut; ++i) vf[t][i] = zero_frag();
    // first row; rows that are there; some query does not see all of them; logits are to be hidden yet
    struct Step { int row; unsigned live; bool edge, shown; };
    Step before{0, 0, true, false}, old{0, 0, false, false};   // of s[1 - cur] and of vf: first of none, with values that are anything

    const unsigned k_base = col * St::kRowBytes + 16 * (half ^ St::key(col));
    const int v_row = 4 * half + lane % 16 / 4;
    const unsigned v_base = v_row * St::kRowBytes + 16 * ((2 * (lane / 16 % 2) + lane % 4 / 2) ^ St::value(v_row)) + 8 * (lane % 2);
    const auto lds_frag = [](unsigned at) __attribute__((always_inline)) { return *(const __attribute__((address_space(3))) frag_t*)(uintptr_t)at; };
    const auto value_frag = [&](unsigned at, int t, int i) __attribute__((always_inline)) {   // rows 16 t .. 16 t + 15 of a step
        const s16x4_t x = read_transposed(((v_base + at) ^ (64 * i)) + 16 * t * St::kRowBytes);
        const s16x4_t y = read_transposed(((v_base + at) ^ (64 * i)) + (16 * t + 8) * St::kRowBytes);
        return __builtin_bit_cast(frag_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Outputs.  Those of the largest tiles are held in the accumulation registers, which the compiler would not do beside logits that
    // the vector ALU reads: their products are written out, and so are the waits that it would place.  A product's operands
    // come two instructions before it at least, its results 18 after it (the build looks whether the first holds in what was
    // compiled, and refuses it otherwise).
    constexpr bool kAcc = D == 128 && kQ == 2;
    const auto add_out = [&](f32x16_t& x, const frag_t& v, const frag_t& w, auto apart) __attribute__((always_inline)) {
        if constexpr (kAcc && decltype(apart)::value) asm volatile("s_nop 1");
        if constexpr (kAcc) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(x) : "v"(v), "v"(w));
        else mma<T>(x, v, w);
    };
    const auto settle_weights = [&]() __attribute__((always_inline)) { if constexpr (kAcc) asm volatile("s_nop 1" ::: "memory"); };
    const auto settle_out = [&]() __attribute__((always_inline)) {
        if constexpr (kAcc)
#pragma unroll
            for (int c = 0; c < kQ; ++c)
                asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3" : "+a"(o[c][0]), "+a"(o[c][1]), "+a"(o[c][2]), "+a"(o[c][kOut - 1]));
    };
    // which of a step's rows 4 half + (0..3) + 8 (0..3) the lane's query sees, bit acc_row(r, 0)
    const auto seen = [&](const Step& st, int c) __attribute__((always_inline)) {
        const int lane = lane_here(), half = lane / 32, left = sees(query(c, lane % 32).token) - st.row;       // (formed anew, as below)
        return ((left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1) & st.live) >> (4 * half);
    };
    const auto hide = [&](f32x16_t (&x)[kQ], const Step& st) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
            const unsigned bits = seen(st, c);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int keep = __builtin_amdgcn_sbfe(bits, acc_row(r, 0), 1);
                x[c][r] = __int_as_float((__float_as_int(x[c][r]) & keep) | (kMinusInf & ~keep));
            }
        }
    };
    // Where some query does not see a row, the row's value counts 0 times: an infinity or NaN there must not.  It is taken out of
    // the products (hardly ever there), and a second product says which queries see one.
    const auto take_out = [&](const Step& st) __attribute__((always_inline)) {
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        typedef unsigned short u16x8_t __attribute__((ext_vector_type(8)));
        s16x8_t up = 0;
        u16x8_t down = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
                up = __builtin_elementwise_max(up, __builtin_bit_cast(s16x8_t, vf[t][i]));
                down = __builtin_elementwise_max(down, __builtin_bit_cast(u16x8_t, vf[t][i]));
            }
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) odd |= up[e] >= 0x7f80 || down[e] >= 0xff80;
        if (!rare(__any(odd))) return;
        settle_out();
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
            const unsigned bits = seen(st, c);
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
                f32x16_t count = zero_acc();
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8_t x = __builtin_bit_cast(bf16x8_t, vf[t][i]);
                    bf16x8_t not_finite, sees;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        not_finite[e] = (bf16_t)(fabsf((float)x[e]) < INFINITY ? 0.f : 1.f);
                        sees[e] = (bf16_t)((bits >> acc_row(8 * t + e, 0)) & 1 ? 1.f : 0.f);
                    }
                    mma<T>(count, __builtin_bit_cast(frag_t, not_finite), __builtin_bit_cast(frag_t, sees));
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) o[c][i][r] = count[r] > 0.f ? NAN : o[c][i][r];
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
                bf16x8_t x = __builtin_bit_cast(bf16x8_t, vf[t][i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fabsf((float)x[e]) < INFINITY ? x[e] : (bf16_t)0.f;
                vf[t][i] = __builtin_bit_cast(frag_t, x);
            }
    };
    // The reference m stays where it is while the weights' sum has room: a row's weights are relative to it, and nothing is lost by
    // their size.  Else it goes up to the largest logit, and the step's weights are formed again.  (A reference that is NaN makes a sum
    // that has none: the first one is found this way.)
    constexpr float kRoom = 0x1p30f;
    const auto raise = [&](const f32x16_t (&x)[kQ], frag_t (&w)[kQ][2], float (&sum)[kQ]) __attribute__((always_inline)) {
        float shrink[kQ];
        bool shrinks = false;
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
            float top = x[c][0];
#pragma unroll
            for (int r = 1; r < 16; ++r) top = fmaxf(top, x[c][r]);
            top = fmaxf(m[c], halves_max(top) * a.scale_log2e);
            const bool set = m[c] > -INFINITY, full = halves_max(sum[c] <= kRoom ? 0.f : 1.f) > 0.f;
            const float m_new = !full ? m[c] : top > -INFINITY ? top : NAN, ref = m_new > -INFINITY ? m_new : 0.f;
            shrink[c] = set ? exp2_fast(m[c] - ref) : 1.f;     // (what there is of a query without a reference is 0)
            shrinks |= full && set;
            m[c] = m_new;
            sum[c] = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                bf16x8_t y;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = exp2_fast(__builtin_fmaf(x[c][8 * t + e], a.scale_log2e, -ref));
                    sum[c] += z;
                    y[e] = (bf16_t)z;
                }
                // (into the registers that hold the others: else every turn would move the one or the other)
                const frag_t z = __builtin_bit_cast(frag_t, y);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    int to = w[c][t][e];
                    asm volatile("v_mov_b32 %0, %1" : "+v"(to) : "v"(z[e]));
                    w[c][t][e] = to;
                }
            }
        }
        if (rare(__any(shrinks))) {
            settle_out();
#pragma unroll
            for (int c = 0; c < kQ; ++c) {
                l[c] *= shrink[c];
#pragma unroll
                for (int i = 0; i < kOut; ++i) o[c][i] *= shrink[c];
            }
        }
    };

    // One turn: the products of step n (keys at k_at) go to s[cur], the weights of step n - 1 come from s[1 - cur], the values of
    // step n - 2 are in vf, and those of step n - 1 (at v_at) take their place.
    constexpr int kPv = 2 * kOut * kQ, kQk = kFrags * kQ, kSlots = kPv + kQk, kElems = 16 * kQ;
    const auto begin = [&](f32x16_t (&x)[kQ], unsigned live) __attribute__((always_inline)) {
        const unsigned gone = ~live >> (4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float y = __int_as_float(__builtin_amdgcn_sbfe(gone, acc_row(r, 0), 1) & kMinusInf);
#pragma unroll
            for (int c = 0; c < kQ; ++c) x[c][r] = y;
        }
    };
    const auto first_turn = [&](unsigned live, unsigned k_at) __attribute__((always_inline)) {              // products alone
        if constexpr (kSome) begin(s[0], live);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const frag_t x = lds_frag((k_base + k_at) ^ (32 * f));
#pragma unroll
            for (int c = 0; c < kQ; ++c) {
                if (f == 0 && !kSome) mma_first<T>(s[0][c], x, qf[c][f]);
                else mma<T>(s[0][c], x, qf[c][f]);
            }
        }
    };
    const auto turn = [&](auto cur_, unsigned live, unsigned k_at, unsigned v_at) __attribute__((always_inline)) {
        constexpr int cur = decltype(cur_)::value;
        if constexpr (kSome) begin(s[cur], live);
        settle_weights();
        float sum[kQ], y[kElems];
#pragma unroll
        for (int c = 0; c < kQ; ++c) sum[c] = 0.f;
        const auto element = [&](int e) __attribute__((always_inline)) {
            if (e < kElems) y[e] = __builtin_fmaf(s[1 - cur][e / 16][e % 16], a.scale_log2e, -m[e / 16]);
            if (e >= 1 && e - 1 < kElems) y[e - 1] = exp2_fast(y[e - 1]);
            if (e >= 2 && e - 2 < kElems) {
                sum[(e - 2) / 16] += y[e - 2];
                if (e % 2 == 1) {
                    const int c = (e - 2) / 16, t = (e - 2) % 16 / 8, i = (e - 2) % 8 / 2;
                    typedef bf16_t pair_t __attribute__((ext_vector_type(2)));
                    p[1 - cur][c][t][i] = __builtin_bit_cast(int, pair_t{(bf16_t)y[e - 3], (bf16_t)y[e - 2]});
                }
            }
        };
#pragma unroll
        for (int n = 0; n < kPv; ++n) {
            const int t = n / (kOut * kQ), i = n / kQ % kOut, c = n % kQ;
            add_out(o[c][i], vf[t][i], p[cur][c][t], std::false_type{});
            if (n >= kPv - kFrags) kf[n - (kPv - kFrags)] = lds_frag((k_base + k_at) ^ (32 * (n - (kPv - kFrags))));
#pragma unroll
            for (int e = n * kElems / kSlots; e < (n + 1) * kElems / kSlots; ++e) element(e);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < kQk; ++n) {
            const int f = n / kQ, c = n % kQ;
            if (f == 0 && !kSome) mma_first<T>(s[cur][c], kf[f], qf[c][f]);
            else mma<T>(s[cur][c], kf[f], qf[c][f]);
            constexpr int kV = 2 * kOut;
#pragma unroll
            for (int x = n; x < min(n + 1, kV); ++x) vf[x / kOut][x % kOut] = value_frag(v_at, x / kOut, x % kOut);
#pragma unroll
            for (int e = (n + kPv) * kElems / kSlots; e < (n + kPv + 1) * kElems / kSlots; ++e) element(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        element(kElems);
        element(kElems + 1);
        const float all = kQ == 2 ? sum[0] + sum[kQ - 1] : sum[0];
        if (rare(__builtin_amdgcn_ballot_w64(!(all <= kRoom)) != 0)) raise(s[1 - cur], p[1 - cur], sum);
#pragma unroll
        for (int c = 0; c < kQ; ++c) l[c] += sum[c];
    };

    // Stages come last rows first.  One is in flight while one is worked on; rows of pages are found four stages at a time.
    //
    // The compiler does not see that wait_vmem ends the queries' loads.  It takes them for under way on every turn and waits for all
    // loads before the first product of a stage that reads them: the keys that the stage has asked for at its begin have the time
    // of one turn's products of weights and values; the values, asked for in its second turn, have until the next stage.  (Where waves
    // share a tile, the keys and values of every next step.)
    const int first_batch = (hi - 1) / kBatch;
    if constexpr (kPaged) {
        if (hi > lo) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int trip = 0; trip < 3; ++trip) {
                    look_up(first_batch - i, trip);
                    wait_vmem<0>();
                }
        }
        __syncthreads();
    }
    int kbuf = 0, vbuf = 0;
    unsigned v_prev = v_lds;                                   // values of the step before (any, where there is none)
    if (hi > lo) {
        load_rows(std::false_type{}, hi * kKv - kRowsOfLoad, k_lds);
        load_rows(std::true_type{}, hi * kKv - kRowsOfLoad, v_lds);
    }
    const bool works = r0 < n_rows;
    bool begun = false;
    int it = hi - 1;
    const auto stage = [&](auto top_) __attribute__((always_inline)) {
        constexpr bool kTop = decltype(top_)::value;           // some query may not see all of the rows at hand
        int vnext = vbuf == 2 ? 0 : vbuf + 1;
        wait_vmem<0>();
        if constexpr (kS == 1) {
            __syncthreads();
            if (it > lo) load_rows(std::false_type{}, (it - 1) * kKv, k_lds + (kbuf ^ 1) * kLoadBytes);
        }
        unsigned long long live = ~0ull;
        if constexpr (kPaged) {
            live = live_of[it % kHold];
            live = ((unsigned long long)(unsigned)scalar((int)(live >> 32)) << 32) | (unsigned)scalar((int)live);
            if (it / kBatch < first_batch) {
                const int trip = kBatch - 1 - it % kBatch;
                if (trip == 0) look_up(it / kBatch - 1, 0);
                else if (trip == 1) look_up(it / kBatch - 1, 1);
                else if (trip == 2) look_up(it / kBatch - 1, 2);
            }
        }
        const auto load_values = [&]() __attribute__((always_inline)) {
            if (kS == 1 && it > lo) load_rows(std::true_type{}, (it - 1) * kKv, v_lds + vnext * kLoadBytes);
        };
        if (works && (!kTop || it * kKv < lim_max)) {
#pragma unroll
            for (int j = 1; j >= 0; --j) {
                if constexpr (kS > 1) {
                    // the values that the last turn read lay where the next ones go, and nothing has waited for them yet (the build
                    // looks whether every way to these loads has)
                    wait_lds_reads();
                    wait_vmem<0>();
                    vnext = vbuf == 2 ? 0 : vbuf + 1;
                    if (j == 1 || it > lo) {
                        load_rows(std::false_type{}, it * kKv + 32 * j - 32, k_lds + (kbuf ^ 1) * kLoadBytes);
                        load_rows(std::true_type{}, it * kKv + 32 * j - 32, v_lds + vnext * kLoadBytes);
                    }
                }
                if (j == 0) load_values();             // (a stage's loads in two parts: a burst of them holds the wave up)
                const unsigned here = (unsigned)(live >> (32 * j)), k_at = k_lds + kbuf * kLoadBytes + (kS > 1 ? 0 : 32 * j * St::kRowBytes);
                // (a step without a live row holds copies of one of the stage's other step, and that one some query may not see)
                const bool edge = kTop && (it * kKv + 32 * j + 32 > lim_min || (kPaged && here == 0 && it * kKv + kKv > lim_min));
                const Step now{it * kKv + 32 * j, here, edge, edge || (kPaged && !kSome && here != ~0u)};
                if (rare(before.shown)) hide(j == 1 ? s[1] : s[0], before);
                if constexpr (kTop) if (rare(old.edge)) take_out(old);
                if (kTop && j == 1 && !begun) {
                    first_turn(here, k_at);
                    begun = true;
                } else if (j == 1) turn(ic<0>{}, here, k_at, v_prev);
                else turn(ic<1>{}, here, k_at, v_prev);
                v_prev = v_lds + vbuf * kLoadBytes + (kS > 1 ? 0 : 32 * j * St::kRowBytes);
                old = before;
                before = now;
                if constexpr (kS > 1) { kbuf ^= 1; vbuf = vnext; }
            }
        }
        else load_values();
        if constexpr (kS == 1) { kbuf ^= 1; vbuf = vnext; }
    };
    // the first stage and those that some query does not see whole, and one more for what is under way; then those that need no look
    const int whole = min(lim_min / kKv, hi) - 1;
    for (; it >= lo && it >= whole; --it) stage(std::true_type{});
    for (; it >= lo; --it) stage(std::false_type{});

    // the last two steps' ends: weights of s[1], values of vf and of v_prev
    if (begun) {
        if (before.shown) hide(s[1], before);
        if (old.edge) take_out(old);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int c = 0; c < kQ; ++c) add_out(o[c][i], vf[t][i], p[0][c][t], std::true_type{});
        float sum[kQ];
#pragma unroll
        for (int c = 0; c < kQ; ++c) sum[c] = INFINITY;        // (the weights are formed here)
        raise(s[1], p[1], sum);
#pragma unroll
        for (int c = 0; c < kQ; ++c) l[c] += sum[c];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kOut; ++i) vf[t][i] = value_frag(v_prev, t, i);
        if (before.edge) take_out(before);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int c = 0; c < kQ; ++c) add_out(o[c][i], vf[t][i], p[1][c][t], std::true_type{});
    }
    settle_out();

#pragma unroll
    for (int c = 0; c < kQ; ++c) m[c] = m[c] > -INFINITY ? m[c] : -INFINITY;
    if constexpr (kS > 1) {
        // the parts' results, where their rings were
        typedef float row_t[D + 4];
        row_t* const mine = reinterpret_cast<row_t*>(&rings[part][0][0]);
        static_assert(5 * kLoadBytes >= 32 * (int)sizeof(row_t), "rows of a part");
        const float total = halves_sum(l[0]);
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4_t*>(&mine[col][32 * i + acc_row(r, half)]) = f32x4_t{o[0][i][r], o[0][i][r + 1], o[0][i][r + 2], o[0][i][r + 3]};
        if (half == 0) { mine[col][D] = m[0]; mine[col][D + 1] = total; }
        __syncthreads();
        for (int x = threadIdx.x; x < 32 * (D / 4); x += 64 * kS) {
            const int at = x / (D / 4), d = x % (D / 4) * 4, row = r0 + at;
            if (row >= n_rows) break;
            const auto of = [&](int w) { return reinterpret_cast<const row_t*>(&rings[w][0][0])[at]; };
            float top = of(0)[D];
#pragma unroll
            for (int w = 1; w < kS; ++w) top = fmaxf(top, of(w)[D]);
            const float ref = top > -INFINITY ? top : 0.f;
            float sum = 0.f;
            f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kS; ++w) {
                const float f = exp2_fast(of(w)[D] - ref);
                sum += f * of(w)[D + 1];
                y += f * *reinterpret_cast<const f32x4_t*>(&of(w)[d]);
            }
            const int tok = row / a.group, qh = head * a.group + row - tok * a.group;
            const long long q_token = seq.q_first + tok;
            if (a.splits > 1) {
                const long long to = (q_token * a.kv_heads * a.group + qh) * a.splits + blockIdx.y;
                *reinterpret_cast<f32x4_t*>(a.part_o + to * D + d) = y;
                if (d == 0) { a.part_ml[2 * to] = top; a.part_ml[2 * to + 1] = sum; }
                continue;
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T* out = reinterpret_cast<T*>(a.out) + qh * a.o_sh + (a.q_start ? q_token * a.o_sn : b * a.o_sb + tok * a.o_sn) + d;
            store4(out, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv, a.o_wide);
            if (a.lse && d == 0) a.lse[(a.q_start ? q_token : b * a.l_sb + tok) + qh * a.l_sh] = (ref + log2_fast(sum)) * 0.6931471805599453f;
        }
        return;
    }

    // ---- the lane's queries: columns 32 i + acc_row(r, half)  (all that is derived from the lane's number is formed anew: nothing of
    // it is held through the loops)
    const int lane2 = lane_here(), col2 = lane2 % 32, half2 = lane2 / 32;
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
        const float total = halves_sum(l[c]);
        const Query at = query(c, col2);
        const bool here = r0 + 32 * c + col2 < n_rows;
        const float ref = m[c] > -INFINITY ? m[c] : 0.f;
        const long long q_token = seq.q_first + at.token;
        if (a.splits > 1) {
            if (!here) continue;
            const long long to = (q_token * a.kv_heads * a.group + at.head) * a.splits + split;
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<f32x4_t*>(a.part_o + to * D + 32 * i + acc_row(r, half2)) = f32x4_t{o[c][i][r], o[c][i][r + 1], o[c][i][r + 2], o[c][i][r + 3]};
            if (half2 == 0) { a.part_ml[2 * to] = m[c]; a.part_ml[2 * to + 1] = total; }
            continue;
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;    // (NaN stays)
        T* out = reinterpret_cast<T*>(a.out) + at.head * a.o_sh + (a.q_start ? q_token * a.o_sn : b * a.o_sb + at.token * a.o_sn);
        // eight neighbouring elements a lane: four of its own and the four that the lane 32 away has
        frag_t pieces[kOut][2];
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    typedef bf16_t pair_t __attribute__((ext_vector_type(2)));
                    const int r = 8 * q + 2 * x;
                    const pair_t even{(bf16_t)(o[c][i][r] * inv), (bf16_t)(o[c][i][r + 1] * inv)};
                    const pair_t odd{(bf16_t)(o[c][i][r + 4] * inv), (bf16_t)(o[c][i][r + 5] * inv)};
                    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, even), __builtin_bit_cast(unsigned, odd), false, false);
                    pieces[i][q][x] = (int)both[0];
                    pieces[i][q][2 + x] = (int)both[1];
                }
        if (!here) continue;
        out += 8 * half2;
        if (a.o_wide) {
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) *reinterpret_cast<frag_t*>(out + 32 * i + 16 * q) = pieces[i][q];
        } else {
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const bf16x8_t x = __builtin_bit_cast(bf16x8_t, pieces[i][q]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[32 * i + 16 * q + e] = x[e];
                }
        }
        if (a.lse && half2 == 0) a.lse[(a.q_start ? q_token : b * a.l_sb + at.token) + at.head * a.l_sh] = (ref + log2_fast(total)) * 0.6931471805599453f;
    }
}

// ---- joining

// A thread has four columns of a query's output.

template <typename T, int D, bool kPaged>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a)
{
    constexpr int kLanes = D / 4;
    const long long row = (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;     // (token, q-head)
    const int d = threadIdx.x % kLanes * 4;
    const int q_heads = a.kv_heads * a.group;
    const long long q_token = row / q_heads;
    const int q_head = (int)(row - q_token * q_heads);
    if (q_token >= a.q_tokens) return;
    int b = 0, token = 0;
    if (!a.q_start) {
        b = (int)(q_token / a.q_rows);
        token = (int)(q_token - (long long)b * a.q_rows);
        if (token >= sequence<kPaged>(a, b).n) return;
    } else {
        // (rows of no sequence stay as they are)
        bool found = false;
        for (; b < a.batch && !found; ++b) {
            const Seq s = sequence<kPaged>(a, b);
            found = q_token >= s.q_first && q_token < s.q_first + s.n;
        }
        if (!found) return;
    }
    const long long at = row * a.splits;
    float m = -INFINITY;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[2 * (at + s)]);
    const float ref = m > -INFINITY ? m : 0.f;
    float l = 0.f;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
        const float f = exp2_fast(a.part_ml[2 * (at + s)] - ref);
        l += f * a.part_ml[2 * (at + s) + 1];
        x += f * *reinterpret_cast<const f32x4_t*>(a.part_o + (at + s) * D + d);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = reinterpret_cast<T*>(a.out) + q_head * a.o_sh + (a.q_start ? q_token * a.o_sn : b * a.o_sb + token * a.o_sn) + d;
    store4(out, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv, a.o_wide);
    if (a.lse && d == 0) a.lse[(a.q_start ? q_token : b * a.l_sb + token) + q_head * a.l_sh] = (ref + log2_fast(l)) * 0.6931471805599453f;
}

// ---- launches

// How a call is cut: rows of a block (256, 64 a wave; 128 or 64, 32 a wave; 32, whose waves share the rows of keys and values), and
// blocks that share a tile's rows of keys and values.  It is what an estimate of the time (us) finds least.  A compute unit takes
// `unit` for 32 query rows by 64 rows of keys and values where it has as many blocks as fit; a block alone takes `stage` for 64
// rows of them, and no call is shorter than its longest block; a join is a launch and its traffic.  The figures are those of prompts
// of 77 to 8192 tokens, each size measured with each choice (us; waves of 32 rows):
//     8 q-heads on 8, D 128, 2048 tokens      1: 26.9   2, split in 2: 34.9
//     8 q-heads on 2, D 64, 4096 tokens       1: 34.9   2: 44.9
//     64 tokens behind 8128                   1, split in 8: 27.2   16: 30.4
//     32 q-heads on 8, D 128, 2048 tokens     2: 51   4: 52   8: 63
//     the same, 4096 tokens                   4: 144   8: 152   (from 8192 on 8 waves' rows are best: 0.21 against 0.27 a unit)
// Where two choices are near each other the estimate may take the other.
PromptPlan plan_prompt(long long sequences, long long rows, long long all_rows, int kv_heads, int group, int head_dim, long long most, bool paged, bool f32)
{
    PromptPlan best{};
    const auto tiles = [&](int waves) {
        const int tile = 32 * waves;
        const long long by_sequence = sequences * ((rows + tile - 1) / tile), together = (all_rows + tile - 1) / tile + sequences;
        return by_sequence < together ? by_sequence : together;
    };
    if (f32) {      // matrix products bound it: two waves a block, and blocks for two waves a SIMD
        best.waves = 2;
        best.tiles = tiles(2);
        best.splits = (int)std::max(1ll, std::min({1024 / (best.tiles * kv_heads), most / 128, 8ll}));
        return best;
    }
    struct Cost { int waves, fit, fit_paged; double unit, stage, begin; };
    static constexpr Cost kWide[] = {{8, 1, 1, 0.21, 1.7, 11.}, {4, 2, 1, 0.27, 1.2, 5.9}, {2, 2, 1, 0.32, 1.2, 5.3}, {1, 2, 1, 0.42, 0.62, 7.4}};     // head size 128
    static constexpr Cost kNarrow[] = {{8, 2, 2, 0.13, 1.1, 11.}, {4, 3, 3, 0.19, 0.66, 5.7}, {2, 4, 3, 0.21, 0.62, 5.3}, {1, 2, 1, 0.25, 0.2, 6.8}};    // 64
    const double stages = (double)((most + 63) / 64), seen = 1. - std::min(1., (double)rows / group / most) / 2;         // of them by a query
    double least = 0.;
    for (const Cost& c : head_dim == 128 ? kWide : kNarrow) {
        const long long n = tiles(c.waves);
        for (int splits = 1; splits <= 16 && (splits == 1 || (most >= 256 * splits && all_rows * kv_heads <= 1 << 22)); splits *= 2) {
            const double blocks = (double)n * kv_heads * splits;
            const double whole = (double)all_rows / 32 * kv_heads * stages * seen * c.unit / 256;
            const int fit = paged ? c.fit_paged : c.fit;
            const double crowd = std::min((double)fit, blocks / 256), stage = std::max(c.stage, c.unit * c.waves * crowd);
            const double longest = (stages / splits + 1) * stage;
            const double rounds = std::ceil(blocks / (256. * fit)) * (stages * seen / splits + 1) * stage;
            const double join = splits > 1 ? 5. + (double)all_rows * kv_heads * splits * head_dim * 8 / 3e6 : 0.;
            const double time = std::max({whole, longest, rounds}) + c.begin + join;
            if (best.waves == 0 || time < least) {
                least = time;
                best.waves = c.waves;
                best.splits = splits;
                best.tiles = n;
            }
        }
    }
    return best;
}

namespace {
template <int D, bool kPaged, bool kSome>
void launch_tiles(const PromptArgs& a, int waves, dim3 grid, hipStream_t st)
{
    constexpr int kS = D == 64 ? 4 : 2;
    if (waves == 8) prompt_kernel<D, kPaged, kSome, 2, 4, 1><<<grid, 256, 0, st>>>(a);
    else if (waves == 4) prompt_kernel<D, kPaged, kSome, 1, 4, 1><<<grid, 256, 0, st>>>(a);
    else if (waves == 2) prompt_kernel<D, kPaged, kSome, 1, 2, 1><<<grid, 128, 0, st>>>(a);
    else prompt_kernel<D, kPaged, kSome, 1, 1, kS><<<grid, 64 * kS, 0, st>>>(a);
}

template <typename T, int D, bool kPaged>
hipError_t launch(PromptArgs a, const PromptPlan& plan, hipStream_t st)
{
    a.page_shift = 0;
    while (1 << a.page_shift < a.page_size) ++a.page_shift;
    a.page_magic = kPaged ? (unsigned)(((1ull << (31 + a.page_shift)) + a.page_size - 1) / a.page_size) : 0;
    a.splits = plan.splits;
    const dim3 grid((unsigned)(plan.tiles * a.kv_heads), plan.splits);
    if constexpr (sizeof(T) == 2) {
        if (kPaged && a.pos_pages) launch_tiles<D, kPaged, kPaged>(a, plan.waves, grid, st);      // (kSome only with kPaged)
        else launch_tiles<D, kPaged, false>(a, plan.waves, grid, st);
    } else {
        prompt_f32_kernel<D, kPaged><<<grid, 128, 0, st>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        const long long rows = a.q_tokens * a.kv_heads * a.group, per = 256 / (D / 4);
        prompt_join_kernel<T, D, kPaged><<<(unsigned)((rows + per - 1) / per), 256, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e;
}
template <typename T>
hipError_t launch_rows(const PromptArgs& a, const PromptPlan& plan, int head_dim, hipStream_t st)
{
    if (a.page_table) return head_dim == 64 ? launch<T, 64, true>(a, plan, st) : launch<T, 128, true>(a, plan, st);
    return head_dim == 64 ? launch<T, 64, false>(a, plan, st) : launch<T, 128, false>(a, plan, st);
}
}  // namespace

hipError_t launch_prompt(const PromptArgs& a, const PromptPlan& plan, int head_dim, bool f32, hipStream_t st)
{
    return f32 ? launch_rows<float>(a, plan, head_dim, st) : launch_rows<bf16_t>(a, plan, head_dim, st);
}

}  // namespace ems
