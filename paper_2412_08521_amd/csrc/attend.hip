// Attention of one new token per sequence over cached rows: o = sum_t p_t v_t / sum_t p_t with p_t = exp(scale q.k_t - m),
// lse = m + ln sum_t p_t, over the live rows t.  One pass with the running maximum m and sum; work is split over the rows
// and joined.
//
// attend_kernel       a block takes the q-heads of one kv-head, 16 or 32 of them, and a stretch of rows, each wave every
//                     fourth step of it.  A step's rows (32; 16 where a row is 512 bytes) are found a lane each, by page
//                     table and position or by table element, shared through LDS, and read straight into the operands
//                     of the matrix products, whose 16 columns are q-heads:
//                       S^T = K Q^T   lane l: key row l % 16 of a tile, 8 columns at 8 (l / 16) of 32
//                       O^T = V^T P^T lane l: its S^T elements are the right operand as they are (rows 4 (l / 16) + r of
//                                     a tile); the left one is a 16-byte piece of each of those rows, transposed between
//                                     registers (two 16-bit elements a v_perm; float32 needs none)
//                     Probabilities go into the products as the exact sum of three bf16 pieces (a float's 24 digits are three
//                     times eight): the numerator's weights are the denominator's.  Two would leave 2^-17 of a probability,
//                     one 2^-8, as much as the output's own rounding; the third takes at most 1 % of a call's time (us, two /
//                     three: the ragged sequences below 675 / 672, 32 x 8 compact heads of 2048 rows 65.8 / 66.0).
//                     Memory bounds it: the products fill 9 % of the matrix pipes.  12 waves a compute unit keep 16 KB
//                     each in flight; 64 sequences of up to 32768 rows, 8 heads of 128 (4.5 GB): 677 us, 6.6 TB/s.
//                     8-bit rows (C = uint8_t): the codes are widened with the row's power of two by the scaled conversion, which
//                     is exact, in front of the same products; a step's rows are half the bytes.  The same ragged
//                     sequences (2.2 GB): 371 to 374 us, 6.05 TB/s.
//                     Several new tokens (kMany): the columns are tokens x q-heads, 32 of them at most.  8 x 4 tokens behind up
//                     to 8192 rows, 32/8 heads of 128: 44 us, and 78 by the kernel of prompts, whose tiles are 32 rows
//                     of one sequence.
// attend_join_kernel  a sequence that several blocks share: their outputs, weighted by their maxima and sums (5 us, a
//                     launch and three trips).
#include "ems_common.h"
#include "ems_kernels.h"
#include "ems_rows.h"

namespace ems {

namespace {

constexpr int kWaves = 4;
constexpr int kNewRow = -2;      // the row of the new token itself (compact cache)
constexpr int kNoRow = -1;

constexpr int kLook = 32;                 // rows that a wave looks up at a time, a lane each
constexpr int kUnit = kAttendUnit;        // what stretches are counted in: a turn of four waves
static_assert(kUnit == kWaves * kLook, "a turn");

template <typename T, int D> constexpr int kRowBytesOf = D * (int)sizeof(T);

// New tokens of a sequence (kMany: a q-head of a token is a column; else there is one, and it has them all).
__device__ __forceinline__ int fresh_tokens(const AttendArgs& a, int b)
{
    return a.new_len ? min(max(a.new_len[b], 0), a.tokens) : a.tokens;
}

// Rows of a sequence (kMany: none, where it has no new token).  A call of one token a sequence does not ask for counts of them: it
// stands before the first trip (us, asking / not: one sequence of 8 heads of 128, 16384 rows 20.4 / 19.6, 700 rows 9.5 / 9.2).
template <bool kMany>
__device__ __forceinline__ int live_len(const AttendArgs& a, bool table, int b)
{
    if (table) return a.n_tok + 1;
    if constexpr (kMany) if (a.new_len && a.new_len[b] <= 0) return 0;
    const long long most = (long long)a.max_pages * a.page_size;
    return (int)min((long long)max(a.lens[b], 0), most);
}

__device__ __forceinline__ int units_of(int len) { return (len + kUnit - 1) / kUnit; }

// t / page_size: the magic number is 2^(31 + shift) / page_size, rounded up, with 2^shift >= page_size
__device__ __forceinline__ int page_of(const AttendArgs& a, int t) { return (int)(__umulhi(2u * (unsigned)t, a.page_magic) >> a.page_shift); }

// a value that is the same in every lane, for the scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// What lanes of a wave wrote to LDS is for its other lanes, and may be written anew once those have read it.  A wave's LDS
// accesses are carried out in their order; the fence holds the compiler to it and is no instruction.
__device__ __forceinline__ void wave_handover()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Workers share the units of a kv-head's sequences evenly: worker w takes `per` of them, one of the first `more` one more.
struct Share {
    int per, more, workers;
    __device__ __forceinline__ Share(int total, int most) : per(total / most), more(total - per * most), workers(per ? most : more) {}
    __device__ __forceinline__ int first_unit(int w) const { return w * per + min(w, more); }
    __device__ __forceinline__ int worker_of(int unit) const
    {
        const int early = more * (per + 1);
        return unit < early ? unit / (per + 1) : more + (unit - early) / per;
    }
};

// The sequence of a worker's first unit, the units of those before it, its rows, and the worker's units; b = -1: it has none.
struct Stretch { int b, before, len, u, u_end; };
template <bool kMany>
__device__ __forceinline__ Stretch stretch_of(const AttendArgs& a, bool table, int worker)
{
    if (table) {
        const int len = a.n_tok + 1, n = units_of(len);
        const Share share(n * a.batch, a.workers);
        const int u = share.first_unit(worker);
        return {worker < share.workers ? u / n : -1, u / n * n, len, u, share.first_unit(worker + 1)};
    }
    const int lane = threadIdx.x % kWave;
    const int len0 = lane < a.batch ? live_len<kMany>(a, table, lane) : 0, n0 = units_of(len0), sum0 = wave_scan(n0);
    int total = 0;
    for (int i = lane + kWave; i < a.batch; i += kWave) total += units_of(live_len<kMany>(a, table, i));
    total = __builtin_amdgcn_readlane(sum0, 63) + (a.batch > kWave ? __builtin_amdgcn_readlane(wave_scan(total), 63) : 0);
    const Share share(total, a.workers);
    Stretch s{-1, 0, 0, share.first_unit(worker), share.first_unit(worker + 1)};
    if (worker >= share.workers) return s;
    int len = len0, n = n0, sum = sum0;
    for (int b0 = 0;;) {
        const unsigned long long past = __ballot(sum > s.u);
        if (past) {
            const int at = __builtin_ctzll(past);
            s.b = b0 + at;
            s.before = __builtin_amdgcn_readlane(sum - n, at);
            s.len = __builtin_amdgcn_readlane(len, at);
            return s;
        }
        b0 += kWave;
        if (b0 >= a.batch) return s;       // not for lengths that stay as they are
        len = b0 + lane < a.batch ? live_len<kMany>(a, table, b0 + lane) : 0;
        n = units_of(len);
        sum = __builtin_amdgcn_readlane(sum, 63) + wave_scan(n);
    }
}

// Units of the sequences before b, and of all of them.
struct Units { int before, total; };
template <bool kMany>
__device__ __forceinline__ Units count_units(const AttendArgs& a, bool table, int b)
{
    if (table) return {b * units_of(a.n_tok + 1), a.batch * units_of(a.n_tok + 1)};
    const int lane = threadIdx.x % kWave;
    int before = 0, total = 0;
    for (int i = lane; i < a.batch; i += kWave) {
        const int n = units_of(live_len<kMany>(a, table, i));
        total += n;
        before += i < b ? n : 0;
    }
    return {__builtin_amdgcn_readlane(wave_scan(before), 63), __builtin_amdgcn_readlane(wave_scan(total), 63)};
}

template <bool kPast, typename V>
__device__ __forceinline__ V read(const V* p) { return kPast ? __builtin_nontemporal_load(p) : *p; }

// Max or sum over the four lanes l % 16 + 16 n that share a column.
template <bool kMax>
__device__ __forceinline__ float column_reduce(float v)
{
    v = comb<kMax>(v, __shfl_xor(v, 16));
    return comb<kMax>(v, __shfl_xor(v, 32));
}

}  // namespace

// T: queries and output, C: keys and values (T, or the bytes of a cache in 8 bits, whose numbers become bf16 as they go into the
// products, the row's power of two with them).
//
// kMany: several new tokens a sequence, the q-heads of each side by side in the columns (a.group of them): a column's token
// sees rows up to its own.
template <typename T, typename C, int D, bool kTable, int kW, bool kPast, int kQt, bool kSparse, bool kMany = false>
__global__ __launch_bounds__(64 * kW, (kQt == 2 ? 2 : kW == 4 ? 3 : kW / 4)) void attend_kernel(AttendArgs a)
{
    constexpr int kTurn = kW * kLook;                          // rows of a block's turn
    constexpr bool k8 = sizeof(C) == 1;
    constexpr int kTiles = kRowBytesOf<C, D> <= 256 ? 2 : 1;    // 16-row tiles of a step: their keys and values wait in registers
    constexpr int kStep = 16 * kTiles, kSteps = kLook / kStep;
    constexpr int kPieces = D * (int)sizeof(T) / 64;           // 16-byte pieces of a query that a lane reads
    constexpr int kKeyPieces = D * (int)sizeof(C) / 64;        // and of a key row: the same columns
    constexpr int kOut = D / 16;                               // output tiles (16 columns of V each)
    constexpr int kCols = D / 16;                              // columns of V that a lane holds of a row
    constexpr size_t kRowBytes = kRowBytesOf<C, D>;
    // a piece of a value row: kCols columns at kCols col (16-bit elements, bytes), or four at 4 col of every 64 (float32)
    constexpr int kVec = k8 ? kCols / 4 : sizeof(T) == 2 ? kCols / 2 : 4;       // dwords
    constexpr int kParts = sizeof(T) == 2 ? 1 : D / 64;
    typedef int vec_t __attribute__((ext_vector_type(kVec)));
    constexpr int kRing = 128;
    __shared__ __align__(16) int row_of[kW][kSparse ? kRing : 2 * kLook];       // two batches, or a ring of live rows
    __shared__ __align__(16) int scale_of[kW][!k8 ? 4 : kSparse ? kRing : 2 * kLook];       // the rows' powers of two: keys' byte, values' above
    __shared__ __align__(16) float factor_of[kW][2][kTable ? kLook : 4];
    __shared__ __align__(16) float red_o[kW][kQt * kAttendQ][D + 4];
    __shared__ float red_ml[kW][kQt * kAttendQ][2];

    const auto turns_of = [](int n) { return (n + kTurn - 1) / kTurn; };
    const int lane = threadIdx.x % kWave, wave = uniform((int)threadIdx.x / kWave);
    const int col = lane % 16, quad = lane / 16;

    // which stretch: units [u, u_end) of the kv-head's sequences, one after the other; base: units of the sequences before b
    const bool shared = kW == kWaves && a.workers;             // else a block per sequence
    const int head = blockIdx.y, tile = blockIdx.z, worker = shared ? blockIdx.x : 0;
    int b = blockIdx.x, u = 0, u_end = 0, base = 0, len = 0;
    if (shared) {
        const Stretch s = stretch_of<kMany>(a, kTable, worker);
        if (s.b < 0) return;
        b = s.b; base = s.before; len = s.len; u = s.u; u_end = s.u_end;
    }
    const int q0 = tile * kQt * kAttendQ, n_q = min(a.group - q0, kQt * kAttendQ);

    for (;;) {
        const int first = u - base;
        const int fresh = kMany ? fresh_tokens(a, b) : 1;
        const int unit = b * a.kv_heads + head;
        const size_t q_head = (size_t)unit * a.group + q0;                          // = b * Hq + head * group + q0

        // queries: the right operand of the first product
        frag_t qf[kQt][kPieces];
#pragma unroll
        for (int j = 0; j < kQt; ++j) {
            const int qi = kAttendQ * j + col;
            const int token = kMany ? (q0 + qi) / a.heads : 0;
            const T* q = reinterpret_cast<const T*>(a.q) + b * a.q_sb + (kMany ? (long long)(head * a.heads + q0 + qi - token * a.heads) * a.q_sh + token * a.q_sn
                                                                              : (long long)(head * a.group + q0 + qi) * a.q_sh);
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
                qf[j][c] = zero_frag();
                if (qi < n_q && token < fresh) {
                    const T* at = q + (k8 ? 64 * (c / 2) + 16 * quad + 8 * (c % 2) : (4 * c + quad) * (16 / (int)sizeof(T)));
                    if (a.q_wide) qf[j][c] = *reinterpret_cast<const frag_t*>(at);
                    else {
                        struct Elems { T x[16 / sizeof(T)]; } e;
#pragma unroll
                        for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e.x[i] = at[i];
                        qf[j][c] = __builtin_bit_cast(frag_t, e);
                    }
                }
            }
        }

        f32x4_t o[kQt][kOut];
        float m[kQt], l[kQt];                                  // of column `col`; l: this lane's rows only
#pragma unroll
        for (int j = 0; j < kQt; ++j) {
            m[j] = -INFINITY; l[j] = 0.f;
#pragma unroll
            for (int i = 0; i < kOut; ++i) o[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }

        // Rows are looked up a batch of 32 ahead in two trips (the table; the position, or the norms), keys and values are
        // requested a step ahead, as soon as the registers that take them are free.
        const int t_first = first * kTurn + wave * kLook + lane % kLook + (kSparse ? lane / kLook * kTurn : 0);
        int t_end = 0;                                         // set below: the first trip does not wait for the lengths
        struct Look { int row, mask; float norm; int scale; };  // mask: the position; norms of the token and of its row
        const auto table_trip = [&](int t) -> int {
            if constexpr (kTable) return t < a.n_tok ? a.tok_row[(size_t)unit * a.n_tok + t] : kNoRow;
            return t < a.max_pages * a.page_size ? a.page_table[(size_t)b * a.max_pages + page_of(a, t)] : kNoRow;
        };
        const auto row_trip = [&](int t, int entry) -> Look {
            Look r{kNoRow, 0, 0.f, 0};
            if constexpr (kTable) {
                // (the index says which is the new token: a caller's element may hold any number)
                r.row = t == a.n_tok ? kNewRow : (unsigned)entry < (unsigned)a.budget ? entry : kNoRow;
                if (r.row >= 0) {
                    r.norm = a.row_norm[(size_t)unit * a.budget + entry];
                    r.mask = __builtin_bit_cast(int, a.tok_norm[(size_t)unit * a.n_tok + t]);
                }
            } else if (t < t_end && entry >= 0 && entry < a.num_pages) {
                r.row = (entry * a.kv_heads + head - page_of(a, t)) * a.page_size + t;       // t % page_size rows into the page
                if (a.pos_pages) r.mask = a.pos_pages[r.row];
                if constexpr (k8) r.scale = a.k_scale[r.row] | a.v_scale[r.row] << 8;
            }
            return r;
        };
        // The batch's rows to LDS; which of them are live.  Dead rows are read as the first live one, which is in the cache
        // already and whose values may meet their zero weights (row 0 where none is live, whose steps are left out).
        const auto settle = [&](int t, const Look& k, int buf) -> unsigned {
            int row = k.row;
            wave_handover();
            if constexpr (kTable) {
                if (t >= t_end) row = kNoRow;
                if (lane < kLook) factor_of[wave][buf][lane] = row == kNewRow ? 1.f : k.norm > 0.f ? __builtin_bit_cast(float, k.mask) / k.norm : 0.f;
            } else if (k.mask < 0) row = kNoRow;
            const unsigned live = (unsigned)__ballot(row != kNoRow);            // the upper lanes look up what others do
            const int spare = live ? __builtin_amdgcn_readlane(row, __builtin_ctz(live)) : 0;
            if (lane < kLook) row_of[wave][kLook * buf + lane] = row != kNoRow ? row : spare;
            if constexpr (k8) {
                const int other = live ? __builtin_amdgcn_readlane(k.scale, __builtin_ctz(live)) : 0;
                if (lane < kLook) scale_of[wave][kLook * buf + lane] = row != kNoRow ? k.scale : other;
            }
            wave_handover();
            return live;
        };
        const auto address = [&](const void* rows, const void* fresh, int r) -> const char* {
            const char* p = reinterpret_cast<const char*>(rows);
            if constexpr (kTable) {
                p += (size_t)unit * (a.budget + 1) * kRowBytes;
                return r == kNewRow ? reinterpret_cast<const char*>(fresh) + unit * kRowBytes : p + (size_t)(unsigned)r * kRowBytes;
            }
            return p + (size_t)(unsigned)r * kRowBytes;
        };
        frag_t kf[kTiles][kKeyPieces];
        float ks[kTiles], vs[kTiles][4];                       // the rows' powers of two (8 bits)
        const auto load_keys = [&](int buf, int at) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int n = kSparse ? (buf + 16 * i + col) % kRing : kLook * buf + kStep * at + 16 * i + col;
                const char* p = address(a.k, a.k_new, row_of[wave][n]) + 16 * quad;
                if constexpr (k8) ks[i] = scale_of_byte(scale_of[wave][n] & 255);
#pragma unroll
                for (int c = 0; c < kKeyPieces; ++c) kf[i][c] = read<kPast>(reinterpret_cast<const frag_t*>(p + 64 * c));
            }
        };
        vec_t vf[kTiles][4][kParts];                           // rows 16 i + 4 quad + r
        const auto load_values = [&](int buf, int at) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int n = kSparse ? (buf + 16 * i + 4 * quad) % kRing + r : kLook * buf + kStep * at + 16 * i + 4 * quad + r;
                    const char* p = address(a.v, a.v_new, row_of[wave][n]) + 4 * kVec * col;
                    if constexpr (k8) vs[i][r] = scale_of_byte(scale_of[wave][n] >> 8);
#pragma unroll
                    for (int h = 0; h < kParts; ++h) vf[i][r][h] = read<kPast>(reinterpret_cast<const vec_t*>(p + 256 * h));
                }
        };
        // Values of rows that some column does not see count 0 times there: infinities and NaN among them (hardly ever) are taken out of
        // the products, and a product of their own says which columns see one.
        const auto take_out = [&](const unsigned (&seen)[kQt]) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int h = 0; h < kParts; ++h)
#pragma unroll
                        for (int d = 0; d < kVec; ++d) {
                            const unsigned x = (unsigned)vf[i][r][h][d];
                            if constexpr (sizeof(T) == 2) odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
                            else odd |= (x & 0x7f800000u) == 0x7f800000u;
                        }
            if (!__any(odd)) return;
            const auto not_finite = [&](int row, int e) -> bool {        // of the lane's rows, output tile e
                const unsigned x = (unsigned)(sizeof(T) == 2 ? vf[row / 4][row % 4][0][e / 2] : vf[row / 4][row % 4][e / 4][e % 4]);
                return sizeof(T) == 2 ? ((e % 2 ? x >> 16 : x) & 0x7f80u) == 0x7f80u : (x & 0x7f800000u) == 0x7f800000u;
            };
#pragma unroll
            for (int e = 0; e < kOut; ++e)
#pragma unroll
                for (int j = 0; j < kQt; ++j) {
                    f32x4_t count = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (sizeof(T) == 2) {
                        bf16x8_t x, y;
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            x[r] = (bf16_t)(not_finite(r, e) ? 1.f : 0.f);
                            y[r] = (bf16_t)((seen[j] >> (16 * (r / 4) + r % 4)) & 1 ? 1.f : 0.f);
                        }
                        count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, count, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4 * kTiles; ++r)
                            count = __builtin_amdgcn_mfma_f32_16x16x4f32(not_finite(r, e) ? 1.f : 0.f, (seen[j] >> (16 * (r / 4) + r % 4)) & 1 ? 1.f : 0.f, count, 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[j][e][r] = count[r] > 0.f ? NAN : o[j][e][r];
                }
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int h = 0; h < kParts; ++h)
#pragma unroll
                        for (int d = 0; d < kVec; ++d) {
                            unsigned x = (unsigned)vf[i][r][h][d];
                            if constexpr (sizeof(T) == 2) {
                                if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
                                if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
                            } else if ((x & 0x7f800000u) == 0x7f800000u) x = 0;
                            vf[i][r][h][d] = (int)x;
                        }
        };
        // one step on the rows in kf and vf, which the rows of (next_buf, next_at) then take
        const auto step = [&](unsigned live, int buf, int at, int next_buf, int next_at, int row = 0) {
            live = uniform((int)(kTiles == 2 ? live : live & 0xffff));
            f32x4_t s[kQt][kTiles];
#pragma unroll
            for (int j = 0; j < kQt; ++j)
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    s[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < kPieces; ++c) {
                        if constexpr (sizeof(T) == 2) {
                            frag_t x;
                            if constexpr (k8) x = widen8(kf[i][c / 2][2 * (c % 2)], kf[i][c / 2][2 * (c % 2) + 1], ks[i]);
                            else x = kf[i][c];
                            s[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x),
                                                                              __builtin_bit_cast(bf16x8_t, qf[j][c]), s[j][i], 0, 0, 0);
                        } else {
                            const f32x4_t x = __builtin_bit_cast(f32x4_t, kf[i][c]), y = __builtin_bit_cast(f32x4_t, qf[j][c]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[j][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], s[j][i], 0, 0, 0);
                        }
                    }
                }
            __builtin_amdgcn_sched_barrier(0);
            load_keys(next_buf, next_at);
            __builtin_amdgcn_sched_barrier(0);
            if (live) {                                        // (row 0 may hold anything)
                // logits in units of ln 2, dead rows -inf whatever their products are
                const bool edge = kMany && row + kStep > len - fresh + 1;       // some column does not see all of the rows
                unsigned seen[kQt];                            // rows 16 i + 4 quad + r, bit 16 i + r
#pragma unroll
                for (int j = 0; j < kQt; ++j) {
                    seen[j] = live;
                    if (edge) {
                        const int left = len - fresh + 1 + (q0 + kAttendQ * j + col) / a.heads - row;
                        seen[j] &= left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
                    }
                    seen[j] >>= 4 * quad;
                }
                if constexpr (kMany) if (edge) take_out(seen);
                f32x4_t f[kTiles];
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    f[i] = f32x4_t{a.scale_log2e, a.scale_log2e, a.scale_log2e, a.scale_log2e};
                    if constexpr (kTable) f[i] *= *reinterpret_cast<const f32x4_t*>(&factor_of[wave][buf][kStep * at + 16 * i + 4 * quad]);
                }
#pragma unroll
                for (int j = 0; j < kQt; ++j) {
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < kTiles; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[j][i][r] = (seen[j] >> (16 * i + r)) & 1 ? s[j][i][r] * f[i][r] : -INFINITY;
                            top = fmaxf(top, s[j][i][r]);
                        }
                    const float m_new = fmaxf(m[j], column_reduce<true>(top));
                    const float ref = m_new > -INFINITY ? m_new : 0.f;
                    if (__any(m_new > m[j])) {
                        const float shrink = exp2_fast(m[j] - ref);
                        l[j] *= shrink;
#pragma unroll
                        for (int i = 0; i < kOut; ++i) o[j][i] *= shrink;
                        m[j] = m_new;
                    }
#pragma unroll
                    for (int i = 0; i < kTiles; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) { s[j][i][r] = exp2_fast(s[j][i][r] - ref); l[j] += s[j][i][r]; }
                }
                if constexpr (sizeof(T) == 2) {
                    bf16x8_t piece[kQt][3];
#pragma unroll
                    for (int j = 0; j < kQt; ++j)
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            float p = s[j][r / 4][r % 4];
#pragma unroll
                            for (int n = 0; n < 3; ++n) {
                                piece[j][n][r] = (bf16_t)p;
                                p -= (float)piece[j][n][r];
                            }
                        }
                    const auto value_pair = [&](int row, int d) -> unsigned {              // columns 2 d, 2 d + 1 of one of the lane's rows
                        const auto& x = vf[row / 4][row % 4][0];
                        if constexpr (!k8) return x[d];
                        return __builtin_bit_cast(unsigned, d % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[d / 2], vs[row / 4][row % 4], true)
                                                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[d / 2], vs[row / 4][row % 4], false));
                    };
#pragma unroll
                    for (int e = 0; e < kCols; ++e) {
                        frag_t x;
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            x[d] = __builtin_amdgcn_perm(value_pair(2 * d + 1, e / 2), value_pair(2 * d, e / 2),
                                                         e % 2 ? 0x07060302 : 0x05040100);
#pragma unroll
                        for (int j = 0; j < kQt; ++j)
#pragma unroll
                            for (int n = 0; n < 3; ++n)
                                o[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), piece[j][n], o[j][e], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kTiles; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int h = 0; h < kParts; ++h) {
                                const f32x4_t x = __builtin_bit_cast(f32x4_t, vf[i][r][h]);
#pragma unroll
                                for (int j = 0; j < kQt; ++j)
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        o[j][4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], s[j][i][r], o[j][4 * h + e], 0, 0, 0);
                            }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_values(next_buf, next_at);
            __builtin_amdgcn_sched_barrier(0);
        };

        int entry = table_trip(t_first);
        if (!shared) {
            len = live_len<kMany>(a, kTable, b);
            u_end = turns_of(len);
        }
        const int seq_units = turns_of(len), last = min(u_end - base, seq_units);      // units of this sequence
        t_end = min(last * kTurn, len);
        if constexpr (kSparse) {
            // Live rows only, packed: 64 lanes look up two turns, what is live goes to a ring in LDS, which the steps empty.
            // Behind the last live row stand kStep copies of it, for steps that are not full.
            const int t0 = first * kTurn + wave * kLook, n_batches = t_end > t0 ? (t_end - t0 + 2 * kTurn - 1) / (2 * kTurn) : 0;
            Look next = row_trip(t_first, entry);
            entry = table_trip(t_first + 2 * kTurn);
            int found = 0, batch = 0;
            const auto find = [&](int need) {                  // rows until there are `need`, or no more
                wave_handover();
                while (found < need && batch < n_batches) {
                    const bool on = next.row != kNoRow && next.mask >= 0;
                    const unsigned long long live = __ballot(on);
                    if (live) {
                        const int at = found + __builtin_amdgcn_mbcnt_hi((unsigned)(live >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)live, 0));
                        const int last = __builtin_amdgcn_readlane(next.row, 63 - __builtin_clzll(live));
                        if (on) row_of[wave][at % kRing] = next.row;
                        if (k8 && on) scale_of[wave][at % kRing] = next.scale;
                        found += __builtin_popcountll(live);
                        if (lane < kStep) row_of[wave][(found + lane) % kRing] = last;
                        if constexpr (k8) {
                            const int scale = __builtin_amdgcn_readlane(next.scale, 63 - __builtin_clzll(live));
                            if (lane < kStep) scale_of[wave][(found + lane) % kRing] = scale;
                        }
                    }
                    ++batch;
                    const int t = t_first + 2 * kTurn * batch;
                    next = row_trip(t, entry);
                    entry = table_trip(t + 2 * kTurn);
                }
                wave_handover();
            };
            find(kStep);
            if (found) {
                load_keys(0, 0);
                load_values(0, 0);
#pragma unroll 1
                for (int at = 0; at < found;) {
                    const int n = min(kStep, found - at);
                    at += n;
                    find(at + kStep);
                    step(n == 32 ? ~0u : (1u << n) - 1, 0, 0, min(at, (found - 1) / kStep * kStep), 0);       // (after the last step, its own rows again)
                }
            }
        } else if (t_end > t_first - lane % kLook) {
            // whole batches, and as many steps of the last one as it has rows
            const int rows = t_end - (t_first - lane % kLook), whole = (rows - 1) / kTurn;
            const int n_steps = whole * kSteps + (min(rows - whole * kTurn, kLook) + kStep - 1) / kStep;
            unsigned live = settle(t_first, row_trip(t_first, entry), 0);
            entry = table_trip(t_first + kTurn);
            load_keys(0, 0);
            load_values(0, 0);
            Look next{kNoRow, 0, 0.f, 0};
#pragma unroll 1
            for (int i = 0, t = t_first + kTurn; i < n_steps; ++i) {           // t: the lane's row of the next batch
                const int at = i % kSteps, buf = i / kSteps & 1;
                if (at == 0) {
                    next = row_trip(t, entry);
                    entry = table_trip(t + kTurn);
                }
                const bool turn = at == kSteps - 1;
                const unsigned now = live >> (kStep * at);
                if (turn) {
                    live = settle(t, next, 1 - buf);
                    t += kTurn;
                }
                step(now, buf, at, turn ? 1 - buf : buf, turn ? 0 : at + 1, t_first - lane % kLook + i / kSteps * kTurn + kStep * at);
            }
        }
#pragma unroll
        for (int j = 0; j < kQt; ++j) l[j] = column_reduce<false>(l[j]);

        {
            // the waves' results.  Element r of tile e: column kCols (4 quad + r) + e, or 64 h + 4 (4 quad + r) + e % 4.
            // (The thread's number is taken anew: what is derived from it would hold registers through the loop above.)
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));
            const int col = tid % 16, quad = tid % kWave / 16;
#pragma unroll
            for (int j = 0; j < kQt; ++j) {
                const int q = kAttendQ * j + col;
                if (quad == 0) { red_ml[wave][q][0] = m[j]; red_ml[wave][q][1] = l[j]; }
                if (q < n_q) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int e = 0; e < kOut; e += 4) {
                            const int d = sizeof(T) == 2 ? kCols * (4 * quad + r) + e : 64 * (e / 4) + 4 * (4 * quad + r);
                            *reinterpret_cast<f32x4_t*>(&red_o[wave][q][d]) = f32x4_t{o[j][e][r], o[j][e + 1][r], o[j][e + 2][r], o[j][e + 3][r]};
                        }
                }
            }
            __syncthreads();
            const bool whole = first == 0 && last == seq_units;
            for (int i = tid; i < n_q * (D / 4); i += 64 * kW) {
                const int q = i / (D / 4), d = i % (D / 4) * 4;
                float top = red_ml[0][q][0];
#pragma unroll
                for (int w = 1; w < kW; ++w) top = fmaxf(top, red_ml[w][q][0]);
                const float ref = top > -INFINITY ? top : 0.f;
                float sum = 0.f;
                f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kW; ++w) {
                    const float f = exp2_fast(red_ml[w][q][0] - ref);
                    sum += f * red_ml[w][q][1];
                    x += f * *reinterpret_cast<const f32x4_t*>(&red_o[w][q][d]);
                }
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;                     // (NaN stays)
                    const int token = kMany ? (q0 + q) / a.heads : 0;
                    if (token >= fresh) continue;
                    const long long h = head * a.heads + q0 + q - token * a.heads;
                    T* out = reinterpret_cast<T*>(a.out) + (kMany ? b * a.o_sb + h * a.o_sh + token * a.o_sn : (q_head + q) * D) + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[e] = (T)(x[e] * inv);
                    if (a.lse && d == 0) a.lse[kMany ? b * a.l_sb + h * a.l_sh + token : q_head + q] = (ref + log2_fast(sum)) * 0.6931471805599453f;
                } else {
                    const size_t at = ((((size_t)(q0 + q) / kAttendQ * a.kv_heads + head) * a.workers + worker) * 2 + (first == 0)) * kAttendQ + q % kAttendQ;
                    *reinterpret_cast<f32x4_t*>(a.part_o + at * D + d) = x;
                    if (d == 0) { a.part_ml[at * 2] = top; a.part_ml[at * 2 + 1] = sum; }
                }
            }
            __syncthreads();
        }
        base += seq_units;
        u = base;
        if (u >= u_end || ++b >= a.batch) break;
        len = live_len<kMany>(a, kTable, b);
    }
}

// A block takes join_q q-heads of a sequence; D / 4 lanes take a q-head's columns, and lanes that are left share its workers.
template <typename T, int D, bool kTable, bool kMany>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    constexpr int kLanes = D / 4, kSlots = 256 / kLanes, kAhead = 4;
    __shared__ float red_ml[kSlots][2];
    __shared__ __align__(16) float red_o[kSlots][D];
    const int b = blockIdx.x, head = blockIdx.y, q0 = blockIdx.z * a.join_q;                   // q0: of the group
    const int len = live_len<kMany>(a, kTable, b);
    const size_t q_head = ((size_t)b * a.kv_heads + head) * a.group + q0;
    const int fresh = kMany ? fresh_tokens(a, b) : 1;
    // element c of the block's q-head (column) i, if there is such a token
    const auto put = [&](int i, int c, float x, float lse) {
        const int token = kMany ? (q0 + i) / a.heads : 0;
        if (token >= fresh) return;
        const long long h = head * a.heads + q0 + i - token * a.heads;
        reinterpret_cast<T*>(a.out)[kMany ? b * a.o_sb + h * a.o_sh + token * a.o_sn + c : (long long)(q_head + i) * D + c] = (T)x;
        if (a.lse && c == 0) a.lse[kMany ? b * a.l_sb + h * a.l_sh + token : q_head + i] = lse;
    };
    if (len == 0) {
        for (int i = threadIdx.x; i < a.join_q * D; i += 256) put(i / D, i % D, 0.f, -INFINITY);
        return;
    }
    const Units units = count_units<kMany>(a, kTable, b);
    const Share share(units.total, a.workers);
    const int w0 = share.worker_of(units.before), w1 = share.worker_of(units.before + units_of(len) - 1);
    if (w0 == w1) return;                                      // one worker had all of it

    const int per = kSlots / a.join_q;                         // lane groups of a q-head
    const int slot = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
    const int qi = slot / per, grp = slot % per, q = q0 + qi;
    if (qi < a.join_q) {
        const size_t at = ((size_t)(q / kAttendQ) * a.kv_heads + head) * a.workers;
        float m = -INFINITY, l = 0.f;
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
        for (int w = w0 + grp; w <= w1; w += per * kAhead) {
            float mw[kAhead], lw[kAhead];
            f32x4_t xw[kAhead];
            float top = m;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int v = w + i * per;
                const size_t part = ((at + min(v, w1)) * 2 + (v == w0)) * kAttendQ + q % kAttendQ;
                mw[i] = a.part_ml[part * 2]; lw[i] = a.part_ml[part * 2 + 1];
                xw[i] = *reinterpret_cast<const f32x4_t*>(a.part_o + part * D + d);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (w + i * per > w1) { mw[i] = -INFINITY; lw[i] = 0.f; xw[i] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
                top = fmaxf(top, mw[i]);
            }
            const float ref = top > -INFINITY ? top : 0.f, f = exp2_fast(m - ref);
            l *= f;
            x *= f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const float fw = exp2_fast(mw[i] - ref);
                l += lw[i] * fw;
                x += xw[i] * fw;
            }
            m = top;
        }
        if (d == 0) { red_ml[slot][0] = m; red_ml[slot][1] = l; }
        *reinterpret_cast<f32x4_t*>(&red_o[slot][d]) = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.join_q * D; i += 256) {
        const int s0 = i / D * per, c = i % D;
        float top = red_ml[s0][0];
        for (int g = 1; g < per; ++g) top = fmaxf(top, red_ml[s0 + g][0]);
        const float ref = top > -INFINITY ? top : 0.f;
        float sum = 0.f, y = 0.f;
        for (int g = 0; g < per; ++g) {
            const float f = exp2_fast(red_ml[s0 + g][0] - ref);
            sum += f * red_ml[s0 + g][1];
            y += f * red_o[s0 + g][c];
        }
        put(i / D, c, y * (sum == 0.f ? 0.f : 1.f / sum), (ref + log2_fast(sum)) * 0.6931471805599453f);
    }
}

// Blocks that share a kv-head's q-heads: one takes a tile of 16, or two where there are more, on the same rows (32 kv-heads
// of 20 q-heads, 605 MB: 109 us, and 172 by blocks of one tile each).
static int tiles_of(int group) { return group <= kAttendQ ? 1 : (group + 2 * kAttendQ - 1) / (2 * kAttendQ); }

// Blocks that share the sequences of a kv-head evenly, or 0: a block per sequence.
//
// Sharing costs the join's launch, 5 us, and a share is a whole number of units; a block of its own has one compute unit's
// bandwidth, some 50 GB/s against 6.2 TB/s of all.  So a block per sequence while the longest that the table admits is
// 256 KB of keys and values (us, block per sequence / shared, one sequence of 8 heads, head size 128: 512 rows 10.5 /
// 11.8, 1024 rows 16.0 / 12.1; 4 heads of 64: 512 rows 8.2 / 10.7, 1024 rows 11.2 / 10.6), and up to 1 MB while there is
// a block for every compute unit (32 sequences of 8 heads and 1024 rows 26.9 / 34.8, 2048 rows 49.7 / 58.2; 2048 rows at
// most, lengths spread evenly: 34.6 / 36.1; 64 such sequences 63.3 / 61.0).  At the bounds themselves the two are near each other.
int attend_workers(int batch, int kv_heads, int group, long long max_len, int row_bytes)
{
    const long long columns = (long long)kv_heads * tiles_of(group);
    if (max_len * 2 * row_bytes <= (columns * batch >= 256 ? 1 << 20 : 1 << 18)) return 0;
    // 768 blocks, rounded up: three a compute unit.  (Where there are two tiles of q-heads in a block, in float32 or at head size
    // 128, two fit: a third of the blocks starts after the others.)
    return (int)((768 + columns - 1) / columns);
}

namespace {
template <typename T, typename C, int D, bool kTable, bool kMany = false>
hipError_t launch(AttendArgs a, hipStream_t st)
{
    a.page_shift = 0;
    while (1 << a.page_shift < a.page_size) ++a.page_shift;
    a.page_magic = a.page_table ? (unsigned)(((1ull << (31 + a.page_shift)) + a.page_size - 1) / a.page_size) : 0;
    // q-heads of a join block: as many as it has lanes for, of the divisors of the group that leave two blocks a compute unit
    a.join_q = 1;
    for (int n = 2; n <= 256 / (D / 4); ++n)
        if (a.group % n == 0 && (long long)a.batch * a.kv_heads * (a.group / n) >= 512) a.join_q = n;
    const int tiles = tiles_of(a.group);
    const long long max_len = kTable ? a.n_tok + 1 : (long long)a.max_pages * a.page_size;
    const long long blocks = (long long)a.batch * a.kv_heads * tiles;
    const dim3 grid(a.workers ? a.workers : a.batch, a.kv_heads, tiles);
    constexpr int kWide = kRowBytesOf<T, D> <= 128 ? 16 : 8;
    // Rows that a block alone reads, and more of them than stay in the caches, go past these (us, plain / past: one sequence of 8
    // heads of 128 and 16384 rows 16.6 / 16.4, 32768 28.8 / 27.1, 131072 97.8 / 86.9; 64 ragged sequences of up to 32768
    // 763 / 703).  More than 32 q-heads of a kv-head are several blocks', tokens of a compact cache share rows: these profit from
    // the caches (64 q-heads 62 / 83, a compact cache of 32 x 8 heads and 2048 rows 66 / 70).  The lengths are on the device: what
    // the table admits decides, and a table wider than its sequences costs what it would not have to (32 sequences of 1024
    // rows, 8 heads, 26.3 us by a table of 1024 rows, 31.7 by one of 4096 or 16384).
    const bool past = !kTable && tiles == 1 && blocks * max_len * 2 * kRowBytesOf<C, D> > 80 << 20;
    //
    // Where such a cache has positions its live rows are packed into full steps.  That costs a little where all are live and
    // saves the steps' loads of nothing where few are (us, packed / not: 128 sequences of 1500 rows, 8 heads, 1 % masked 135
    // / 130, 30 % 97 / 99; 157 of 6451, 60 % 300 / 342; float32, 14 of 109374, 20 q-heads a kv-head, 60 % 328 / 604), and
    // a microsecond of a short call.
    //
    // A block per sequence has eight waves (or 16, as the registers allow) where it would need several turns of four, and
    // there is less than two blocks' work for a compute unit (us at 8 heads of 128 and 512 rows, eight waves / four:
    // 16 sequences 11.5 / 12.4, 32 15.2 / 15.8, 64 29.7 / 27.5, 128 56.6 / 50.4).
    if constexpr (kMany) {
        if (a.group > kAttendQ && past) attend_kernel<T, C, D, kTable, kWaves, true, 2, false, true><<<grid, 256, 0, st>>>(a);
        else if (a.group > kAttendQ) attend_kernel<T, C, D, kTable, kWaves, false, 2, false, true><<<grid, 256, 0, st>>>(a);
        else if (past) attend_kernel<T, C, D, kTable, kWaves, true, 1, false, true><<<grid, 256, 0, st>>>(a);
        else attend_kernel<T, C, D, kTable, kWaves, false, 1, false, true><<<grid, 256, 0, st>>>(a);
    } else if (a.group > kAttendQ) {
        if (past && a.pos_pages) attend_kernel<T, C, D, kTable, kWaves, !kTable, 2, !kTable><<<grid, 256, 0, st>>>(a);
        else if (past) attend_kernel<T, C, D, kTable, kWaves, !kTable, 2, false><<<grid, 256, 0, st>>>(a);
        else attend_kernel<T, C, D, kTable, kWaves, false, 2, false><<<grid, 256, 0, st>>>(a);
    } else if (!a.workers && max_len > kUnit && blocks < 512) {
        attend_kernel<T, C, D, kTable, kWide, false, 1, false><<<grid, 64 * kWide, 0, st>>>(a);
    } else if (past && a.pos_pages) {
        attend_kernel<T, C, D, kTable, kWaves, !kTable, 1, !kTable><<<grid, 256, 0, st>>>(a);
    } else if (past) {
        attend_kernel<T, C, D, kTable, kWaves, !kTable, 1, false><<<grid, 256, 0, st>>>(a);
    } else {
        attend_kernel<T, C, D, kTable, kWaves, false, 1, false><<<grid, 256, 0, st>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.workers) {
        attend_join_kernel<T, D, kTable, kMany><<<dim3(a.batch, a.kv_heads, a.group / a.join_q), 256, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e;
}
template <typename T>
hipError_t launch_rows(const AttendArgs& a, hipStream_t st)
{
    if (a.many) return a.head_dim == 64 ? launch<T, T, 64, false, true>(a, st) : launch<T, T, 128, false, true>(a, st);
    if (a.page_table) return a.head_dim == 64 ? launch<T, T, 64, false>(a, st) : launch<T, T, 128, false>(a, st);
    return a.head_dim == 64 ? launch<T, T, 64, true>(a, st) : launch<T, T, 128, true>(a, st);
}
}  // namespace

hipError_t launch_attend(const AttendArgs& a, bool f32, hipStream_t st)
{
    if (a.k_scale) return a.head_dim == 64 ? launch<bf16_t, uint8_t, 64, false>(a, st) : launch<bf16_t, uint8_t, 128, false>(a, st);
    return f32 ? launch_rows<float>(a, st) : launch_rows<bf16_t>(a, st);
}

}  // namespace ems
