// Attention of one new token per sequence over cached rows: o = sum_t p_t v_t / sum_t p_t with p_t = exp(scale q.k_t - m),
// lse = m + ln sum_t p_t, over the live rows t.  One pass with the running maximum m and sum; work is split over the rows
// and joined.
//
// attend_kernel       a block takes a tile of up to 16 q-heads of one kv-head and a stretch of rows, each wave every fourth
//                     step of it.  A step's rows (64 of 16-bit elements, 32 of float32) are found a lane each (page table
//                     and position, or table element), shared through LDS, and read straight into the operands of the
//                     matrix products, whose 16 columns are the q-heads:
//                       S^T = K Q^T   lane l: key row l % 16 of a tile, 8 columns at 8 (l / 16) of 32
//                       O^T = V^T P^T lane l: its S^T elements are the right operand as they are (rows 4 (l / 16) + r of
//                                     a tile); the left one is a 16-byte piece of each of those rows, transposed between
//                                     registers (two 16-bit elements a v_perm; float32 needs none)
//                     Probabilities go into the products as two bf16 pieces, high and rest (2^-17 of a probability is
//                     left out; one piece would leave 2^-9, as much as the output's own rounding).
// attend_join_kernel  a sequence that several blocks share: their outputs, weighted by their maxima and sums.
#include "ems_common.h"
#include "ems_kernels.h"
#include "ems_rows.h"

namespace ems {

namespace {

constexpr int kWaves = 4;
constexpr int kNewRow = -2;      // the row of the new token itself (compact cache)
constexpr int kNoRow = -1;

constexpr int kLook = 64;                 // rows that a wave looks up at a time, a lane each
constexpr int kUnit = kWaves * kLook;     // rows of a block's turn: what stretches are counted in

template <typename T, int D> constexpr int kRowBytesOf = D * (int)sizeof(T);

__device__ __forceinline__ int live_len(const AttendArgs& a, bool table, int b)
{
    if (table) return a.n_tok + 1;
    const long long most = (long long)a.max_pages * a.page_size;
    return (int)min((long long)max(a.lens[b], 0), most);
}

__device__ __forceinline__ int units_of(int len) { return (len + kUnit - 1) / kUnit; }

// a value that is the same in every lane, for the scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x)
{
    return (long long)(unsigned)uniform((int)x) | (long long)uniform((int)(x >> 32)) << 32;
}

// Units of sequences 0..b-1, or of all of them (b = batch); the same in every lane.
__device__ __forceinline__ long long units_before(const AttendArgs& a, bool table, int b)
{
    if (table) return (long long)b * units_of(a.n_tok + 1);
    const int lane = threadIdx.x % kWave;
    long long n = 0;
    for (int i = lane; i < b; i += kWave) n += units_of(live_len(a, table, i));
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) n += __shfl_xor(n, s);
    return uniform(n);
}

// Max or sum over the four lanes l % 16 + 16 n that share a column.
template <bool kMax>
__device__ __forceinline__ float column_reduce(float v)
{
    v = comb<kMax>(v, __shfl_xor(v, 16));
    return comb<kMax>(v, __shfl_xor(v, 32));
}

}  // namespace

template <typename T, int D, bool kTable>
__global__ __launch_bounds__(256, sizeof(T) == 2 && !(kTable && D == 128) ? 3 : 2) void attend_kernel(AttendArgs a)
{
    constexpr int kTiles = kRowBytesOf<T, D> <= 256 ? 2 : 1;    // 16-row tiles of a step: their keys and values wait in registers
    constexpr int kStep = 16 * kTiles, kSteps = kLook / kStep;
    constexpr int kPieces = D * (int)sizeof(T) / 64;           // 16-byte pieces of a key row that a lane reads
    constexpr int kOut = D / 16;                               // output tiles (16 columns of V each)
    constexpr int kCols = D / 16;                              // columns of V that a lane holds of a row
    constexpr size_t kRowBytes = kRowBytesOf<T, D>;
    // a piece of a value row: kCols columns at kCols col (16-bit elements), or four at 4 col of every 64 (float32)
    constexpr int kVec = sizeof(T) == 2 ? kCols / 2 : 4;       // dwords
    constexpr int kParts = sizeof(T) == 2 ? 1 : D / 64;
    typedef int vec_t __attribute__((ext_vector_type(kVec)));
    __shared__ __align__(16) int row_of[kWaves][2][kLook];
    __shared__ __align__(16) float factor_of[kWaves][2][kTable ? kLook : 4];
    __shared__ __align__(16) float red_o[kWaves][kAttendQ][D + 4];
    __shared__ float red_ml[kWaves][kAttendQ][2];

    const int lane = threadIdx.x % kWave, wave = uniform((int)threadIdx.x / kWave);
    const int col = lane % 16, quad = lane / 16;
    const int group_tiles = (a.group + kAttendQ - 1) / kAttendQ;

    // which stretch: units [u, u_end) of the kv-head's sequences, one after the other
    int b, tile, head, worker = 0;
    long long u, u_end, base;                                  // base: units of the sequences before b
    if (a.workers) {
        worker = blockIdx.x % a.workers;
        const int ht = blockIdx.x / a.workers;
        head = ht % a.kv_heads; tile = ht / a.kv_heads;
        const long long total = units_before(a, kTable, a.batch);
        const long long workers = min((long long)a.workers, total);               // none without a unit
        if (worker >= workers) return;
        u = worker * total / workers;
        u_end = (worker + 1) * total / workers;
        base = 0;
        for (b = 0; b < a.batch - 1; ++b) {
            const int n = units_of(live_len(a, kTable, b));
            if (u < base + n) break;
            base += n;
        }
    } else {
        b = blockIdx.x % a.batch;
        const int ht = blockIdx.x / a.batch;
        head = ht % a.kv_heads; tile = ht / a.kv_heads;
        base = 0; u = 0;
        u_end = units_of(live_len(a, kTable, b));
    }
    (void)group_tiles;
    const int q0 = tile * kAttendQ, n_q = min(a.group - q0, kAttendQ);

    do {
        const int len = live_len(a, kTable, b);
        const long long seq_units = units_of(len);
        const long long first = u - base, last = min(u_end - base, seq_units);      // units of this sequence
        const int unit = b * a.kv_heads + head;
        const size_t q_head = (size_t)unit * a.group + q0;                          // = b * Hq + head * group + q0

        // queries: the right operand of the first product
        frag_t qf[kPieces];
        {
            const T* q = reinterpret_cast<const T*>(a.q) + b * a.q_sb + (long long)(head * a.group + q0 + col) * a.q_sh;
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
                qf[c] = zero_frag();
                if (col < n_q) {
                    const T* at = q + (4 * c + quad) * (16 / (int)sizeof(T));
                    if (a.q_wide) qf[c] = *reinterpret_cast<const frag_t*>(at);
                    else {
                        struct Elems { T x[16 / sizeof(T)]; } e;
#pragma unroll
                        for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e.x[i] = at[i];
                        qf[c] = __builtin_bit_cast(frag_t, e);
                    }
                }
            }
        }

        f32x4_t o[kOut];
#pragma unroll
        for (int i = 0; i < kOut; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;                          // of column `col`; l: this lane's rows only

        // Rows are looked up a batch of 64 ahead in two trips (the table; the position, or the norms), keys and values are
        // requested a step ahead, as soon as the registers that take them are free.
        const int t_end = (int)min(last * kUnit, (long long)len);
        const int t_first = (int)(first * kUnit) + wave * kLook + lane;
        const int n_batches = t_end > t_first - lane ? (t_end - (t_first - lane) + kUnit - 1) / kUnit : 0;
        struct Look { int row, mask; float norm; };            // mask: the position; norms of the token and of its row
        const auto table_trip = [&](int t) -> int {
            if constexpr (kTable) return t < a.n_tok ? a.tok_row[(size_t)unit * a.n_tok + t] : t == a.n_tok ? kNewRow : kNoRow;
            return t < t_end ? a.page_table[(size_t)b * a.max_pages + t / a.page_size] : kNoRow;
        };
        const auto row_trip = [&](int t, int entry) -> Look {
            Look r{kNoRow, 0, 0.f};
            if constexpr (kTable) {
                r.row = entry;
                if (entry >= a.budget || entry < kNewRow) r.row = kNoRow;
                if (r.row >= 0) {
                    r.norm = a.row_norm[(size_t)unit * a.budget + entry];
                    r.mask = __builtin_bit_cast(int, a.tok_norm[(size_t)unit * a.n_tok + t]);
                }
            } else if (t < t_end && entry >= 0 && entry < a.num_pages) {
                r.row = (entry * a.kv_heads + head) * a.page_size + t % a.page_size;
                if (a.pos_pages) r.mask = a.pos_pages[r.row];
            }
            return r;
        };
        // the batch's rows to LDS; which of them are live.  Dead rows are read as the first live one, which is in bounds
        // and in the cache already (row 0 where none is live).
        const auto settle = [&](int t, const Look& k, int buf) -> unsigned long long {
            int row = k.row;
            if constexpr (kTable) {
                if (t >= t_end) row = kNoRow;
                factor_of[wave][buf][lane] = row == kNewRow ? 1.f : k.norm > 0.f ? __builtin_bit_cast(float, k.mask) / k.norm : 0.f;
            } else if (k.mask < 0) row = kNoRow;
            const unsigned long long live = __ballot(row != kNoRow);
            const int spare = live ? __builtin_amdgcn_readlane(row, __builtin_ctzll(live)) : 0;
            row_of[wave][buf][lane] = row != kNoRow ? row : spare;
            __builtin_amdgcn_wave_barrier();
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
        frag_t kf[kTiles][kPieces];
        const auto load_keys = [&](int buf, int at) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const char* p = address(a.k, a.k_new, row_of[wave][buf][kStep * at + 16 * i + col]) + 16 * quad;
#pragma unroll
                for (int c = 0; c < kPieces; ++c) kf[i][c] = *reinterpret_cast<const frag_t*>(p + 64 * c);
            }
        };
        vec_t vf[kTiles][4][kParts];                           // rows 16 i + 4 quad + r
        const auto load_values = [&](int buf, int at) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const char* p = address(a.v, a.v_new, row_of[wave][buf][kStep * at + 16 * i + 4 * quad + r]) + 4 * kVec * col;
#pragma unroll
                    for (int h = 0; h < kParts; ++h) vf[i][r][h] = *reinterpret_cast<const vec_t*>(p + 256 * h);
                }
        };
        // one step on the rows in kf and vf, which the rows of (next_buf, next_at) then take
        const auto step = [&](unsigned live, int buf, int at, int next_buf, int next_at) {
            f32x4_t s[kTiles];
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                s[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kPieces; ++c) {
                    if constexpr (sizeof(T) == 2) {
                        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[i][c]),
                                                                       __builtin_bit_cast(bf16x8_t, qf[c]), s[i], 0, 0, 0);
                    } else {
                        const f32x4_t x = __builtin_bit_cast(f32x4_t, kf[i][c]), y = __builtin_bit_cast(f32x4_t, qf[c]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], s[i], 0, 0, 0);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_keys(next_buf, next_at);
            __builtin_amdgcn_sched_barrier(0);
            // logits in units of ln 2, dead rows -inf whatever their products are
            live >>= 4 * quad;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                f32x4_t f = {a.scale_log2e, a.scale_log2e, a.scale_log2e, a.scale_log2e};
                if constexpr (kTable) f *= *reinterpret_cast<const f32x4_t*>(&factor_of[wave][buf][kStep * at + 16 * i + 4 * quad]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][r] = (live >> (16 * i + r)) & 1 ? s[i][r] * f[r] : -INFINITY;
                    top = fmaxf(top, s[i][r]);
                }
            }
            const float m_new = fmaxf(m, column_reduce<true>(top));
            const float ref = m_new > -INFINITY ? m_new : 0.f;
            if (__any(m_new > m)) {
                const float shrink = exp2_fast(m - ref);
                l *= shrink;
#pragma unroll
                for (int i = 0; i < kOut; ++i) o[i] *= shrink;
                m = m_new;
            }
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) { s[i][r] = exp2_fast(s[i][r] - ref); l += s[i][r]; }
            // what stands in a dead row must not meet its zero weight
            constexpr unsigned kMine = kTiles == 2 ? 0x000f000f : 0xf;
            if (!__all((live & kMine) == kMine)) {
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int h = 0; h < kParts; ++h)
#pragma unroll
                            for (int w = 0; w < kVec; ++w) vf[i][r][h][w] = (live >> (16 * i + r)) & 1 ? vf[i][r][h][w] : 0;
            }
            if constexpr (sizeof(T) == 2) {
                bf16x8_t high, rest;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float p = s[r / 4][r % 4];
                    high[r] = (bf16_t)p;
                    rest[r] = (bf16_t)(p - (float)high[r]);
                }
#pragma unroll
                for (int e = 0; e < kCols; ++e) {
                    frag_t x;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        x[j] = __builtin_amdgcn_perm(vf[(2 * j + 1) / 4][(2 * j + 1) % 4][0][e / 2], vf[2 * j / 4][2 * j % 4][0][e / 2],
                                                     e % 2 ? 0x07060302 : 0x05040100);
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), high, o[e], 0, 0, 0);
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), rest, o[e], 0, 0, 0);
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
                            for (int e = 0; e < 4; ++e)
                                o[4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], s[i][r], o[4 * h + e], 0, 0, 0);
                        }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_values(next_buf, next_at);
            __builtin_amdgcn_sched_barrier(0);
        };

        if (n_batches) {
            int entry = table_trip(t_first);
            unsigned long long live = settle(t_first, row_trip(t_first, entry), 0);
            entry = table_trip(t_first + kUnit);
            load_keys(0, 0);
            load_values(0, 0);
            for (int j = 0, t = t_first + kUnit; j < n_batches; ++j, t += kUnit) {          // t: the lane's row of batch j + 1
                const int buf = j & 1;
                const Look next = row_trip(t, entry);
                entry = table_trip(t + kUnit);
#pragma unroll
                for (int i = 0; i < kSteps - 1; ++i) step((unsigned)(live >> (kStep * i)), buf, i, buf, i + 1);
                const unsigned rest = (unsigned)(live >> (kLook - kStep));
                live = settle(t, next, 1 - buf);
                step(rest, buf, kSteps - 1, 1 - buf, 0);
            }
        }
        l = column_reduce<false>(l);

        // the four waves' results.  Element r of tile e: column kCols (4 quad + r) + e, or 64 h + 4 (4 quad + r) + e % 4.
        if (quad == 0) { red_ml[wave][col][0] = m; red_ml[wave][col][1] = l; }
        if (col < n_q) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < kOut; e += 4) {
                    const int d = sizeof(T) == 2 ? kCols * (4 * quad + r) + e : 64 * (e / 4) + 4 * (4 * quad + r);
                    *reinterpret_cast<f32x4_t*>(&red_o[wave][col][d]) = f32x4_t{o[e][r], o[e + 1][r], o[e + 2][r], o[e + 3][r]};
                }
        }
        __syncthreads();
        const bool whole = first == 0 && last == seq_units;
        const size_t part = a.workers ? (((size_t)tile * a.kv_heads + head) * a.workers + worker) * 2 + (first == 0) : 0;
        for (int i = threadIdx.x; i < n_q * (D / 4); i += 256) {
            const int q = i / (D / 4), d = i % (D / 4) * 4;
            float top = red_ml[0][q][0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, red_ml[w][q][0]);
            const float ref = top > -INFINITY ? top : 0.f;
            float sum = 0.f;
            f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = exp2_fast(red_ml[w][q][0] - ref);
                sum += f * red_ml[w][q][1];
                x += f * *reinterpret_cast<const f32x4_t*>(&red_o[w][q][d]);
            }
            if (whole) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;                     // (NaN stays)
                T* out = reinterpret_cast<T*>(a.out) + (q_head + q) * D + d;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (T)(x[e] * inv);
                if (a.lse && d == 0) a.lse[q_head + q] = (ref + log2_fast(sum)) * 0.6931471805599453f;
            } else {
                *reinterpret_cast<f32x4_t*>(a.part_o + (part * kAttendQ + q) * D + d) = x;
                if (d == 0) { a.part_ml[(part * kAttendQ + q) * 2] = top; a.part_ml[(part * kAttendQ + q) * 2 + 1] = sum; }
            }
        }
        __syncthreads();
        base += seq_units;
        u = base;
        ++b;
    } while (u < u_end && b < a.batch);
}

// One block per (sequence, q-head): kGroups groups of D / 4 lanes each take every kGroups-th worker.
template <typename T, int D, bool kTable>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    __shared__ float red_ml[kGroups][2];
    __shared__ __align__(16) float red_o[kGroups][D];
    const int q_heads = a.kv_heads * a.group;
    const int b = blockIdx.x / q_heads, qh = blockIdx.x % q_heads, head = qh / a.group, q = qh % a.group;
    const int len = live_len(a, kTable, b);
    T* out = reinterpret_cast<T*>(a.out) + (size_t)blockIdx.x * D;
    if (len == 0) {
        if (threadIdx.x < D) out[threadIdx.x] = (T)0.f;
        if (a.lse && threadIdx.x == 0) a.lse[blockIdx.x] = -INFINITY;
        return;
    }
    const long long total = units_before(a, kTable, a.batch), base = units_before(a, kTable, b);
    // worker w takes units [w total / workers, (w + 1) total / workers)
    const long long workers = min((long long)a.workers, total);
    const auto worker_of = [&](long long unit) { return (int)(((unit + 1) * workers - 1) / total); };
    const int w0 = worker_of(base), w1 = worker_of(base + units_of(len) - 1);
    if (w0 == w1) return;                                      // one worker had all of it

    const int grp = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
    const size_t at = ((size_t)(q / kAttendQ) * a.kv_heads + head) * a.workers;
    float m = -INFINITY, l = 0.f;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0 + grp; w <= w1; w += kGroups) {
        const size_t part = ((at + w) * 2 + (w == w0)) * kAttendQ + q % kAttendQ;
        const float mw = a.part_ml[part * 2], lw = a.part_ml[part * 2 + 1];
        const f32x4_t xw = *reinterpret_cast<const f32x4_t*>(a.part_o + part * D + d);
        const float m_new = fmaxf(m, mw), ref = m_new > -INFINITY ? m_new : 0.f;
        const float f = exp2_fast(m - ref), fw = exp2_fast(mw - ref);
        l = l * f + lw * fw;
        x = x * f + xw * fw;
        m = m_new;
    }
    if (d == 0) { red_ml[grp][0] = m; red_ml[grp][1] = l; }
    *reinterpret_cast<f32x4_t*>(&red_o[grp][d]) = x;
    __syncthreads();
    if (threadIdx.x >= D) return;
    float top = red_ml[0][0];
#pragma unroll
    for (int g = 1; g < kGroups; ++g) top = fmaxf(top, red_ml[g][0]);
    const float ref = top > -INFINITY ? top : 0.f;
    float sum = 0.f, y = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const float f = exp2_fast(red_ml[g][0] - ref);
        sum += f * red_ml[g][1];
        y += f * red_o[g][threadIdx.x];
    }
    out[threadIdx.x] = (T)(y * (sum == 0.f ? 0.f : 1.f / sum));
    if (a.lse && threadIdx.x == 0) a.lse[blockIdx.x] = (ref + log2_fast(sum)) * 0.6931471805599453f;
}

// Blocks that share the sequences of a kv-head evenly, or 0: a block per sequence.
int attend_workers(int batch, int kv_heads, int group, long long max_len)
{
    if (max_len <= 256) return 0;
    const long long columns = (long long)kv_heads * ((group + kAttendQ - 1) / kAttendQ);
    const long long want = (768 + columns - 1) / columns;      // three blocks a compute unit
    return (int)want;
}

namespace {
template <typename T, int D, bool kTable>
hipError_t launch(const AttendArgs& a, hipStream_t st)
{
    const int tiles = (a.group + kAttendQ - 1) / kAttendQ;
    attend_kernel<T, D, kTable><<<(a.workers ? a.workers : a.batch) * a.kv_heads * tiles, 256, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.workers) {
        attend_join_kernel<T, D, kTable><<<a.batch * a.kv_heads * a.group, 256, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e;
}
template <typename T>
hipError_t launch_rows(const AttendArgs& a, hipStream_t st)
{
    if (a.page_table) return a.head_dim == 64 ? launch<T, 64, false>(a, st) : launch<T, 128, false>(a, st);
    return a.head_dim == 64 ? launch<T, 64, true>(a, st) : launch<T, 128, true>(a, st);
}
}  // namespace

hipError_t launch_attend(const AttendArgs& a, bool f32, hipStream_t st)
{
    return f32 ? launch_rows<float>(a, st) : launch_rows<bf16_t>(a, st);
}

}  // namespace ems
