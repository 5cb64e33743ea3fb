// Attention of many queries: o_i = sum_t p_t v_t / sum_t p_t with p_t = exp(scale q_i.k_t - m), lse_i = m + ln sum_t p_t, over the
// live rows t <= i + m - n that query i of n sees of m rows.  One pass with the running maximum m and sum.
//
// prompt_kernel  a block takes a tile of query rows of one kv-head, the group's q-heads of a token side by side (row token *
//                group + head), 32 rows a wave, and walks the rows of keys and values in stages through LDS that all its
//                waves read:
//                  S^T = K Q^T    32x32 products; a lane holds one query's column, 16 of a tile's 32 rows
//                  O^T = V^T P^T  S^T's registers are the right operand as they are; the left one is read transposed
// prompt_join    a tile whose rows several blocks share: their outputs, weighted by their maxima and sums
#include "ems_common.h"
#include "ems_kernels.h"
#include "ems_rows.h"
#include "ems_stream.h"

namespace ems {

namespace {

constexpr int kNoRow = -1;

// A sequence: its queries, its rows, and where they begin.
struct Seq { int n, m; long long q_first, k_first; };

template <bool kPaged>
__device__ __forceinline__ Seq sequence(const PromptArgs& a, int b)
{
    if constexpr (kPaged) {
        const long long most = (long long)a.max_pages * a.page_size;
        const int n = a.new_len ? min(max(a.new_len[b], 0), a.q_rows) : a.q_rows;
        return {n, (int)min((long long)max(a.lens[b], 0), most), (long long)b * a.q_rows, 0};
    }
    if (!a.q_start) return {a.q_rows, a.k_rows, (long long)b * a.q_rows, 0};
    const int q0 = min(max(a.q_start[b], 0), a.q_rows), q1 = min(max(a.q_start[b + 1], q0), a.q_rows);
    const int k0 = min(max(a.k_start[b], 0), a.k_rows), k1 = min(max(a.k_start[b + 1], k0), a.k_rows);
    return {q1 - q0, k1 - k0, q0, k0};
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

// From global memory to LDS, a piece of 16 bytes a lane, from the wave's address on; wait_vmem counts it.
__device__ __forceinline__ void dma16(const char* from, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(scalar((int)lds)) : "memory", "m0");
}

}  // namespace

template <typename T, int D, bool kPaged, int kW>
__global__ __launch_bounds__(64 * kW, 2) void prompt_kernel(PromptArgs a)
{
    using St = Stage<T, D>;
    constexpr int kKv = St::kRows, kSubs = kKv / 32;
    constexpr int kFrags = Tile<T, D>::kFrags, kOut = D / 32;
    constexpr int kRowsOf = 32 * kW;
    constexpr int kHold = 4;                                   // tiles whose rows are known
    __shared__ __align__(1024) char stage[2][2][St::kBytes];
    __shared__ int row_of[kPaged ? kHold : 1][kKv];
    __shared__ unsigned long long live_of[kPaged ? kHold : 1];

    const int lane = threadIdx.x % kWave, wave = scalar((int)threadIdx.x / kWave);
    const int col = lane % 32, half = lane / 32;
    const int head = blockIdx.x % a.kv_heads;
    int item = blockIdx.x / a.kv_heads, b = 0;
    const int split = blockIdx.y;
    Seq seq{};
    int n_tiles = 0;
    for (; b < a.batch; ++b) {
        seq = sequence<kPaged>(a, b);
        n_tiles = (int)(((long long)seq.n * a.group + kRowsOf - 1) / kRowsOf);
        if (item < n_tiles) break;
        item -= n_tiles;
    }
    if (b == a.batch) return;
    const int tile = n_tiles - 1 - item;                       // the last tiles have the most rows to see
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
        for (int f = 0; f < kFrags; ++f) {
            const T* at = q + (2 * f + half) * (16 / (int)sizeof(T));
            qf[f] = load_piece(at, a.q_wide);
        }
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
        const unsigned long long live = __ballot(r != kNoRow);
        const int spare = live ? __builtin_amdgcn_readlane(r, __builtin_ctzll(live)) : 0;
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
        const int r = 4 * half + lane % 16 / 4;
        if constexpr (sizeof(T) == 2)
            v_base[i] = lds + St::kBytes + r * St::kRowBytes + 16 * ((4 * i + 2 * (lane / 16 % 2) + lane % 4 / 2) ^ St::value(r)) + 8 * (lane % 2);
        else
            v_base[i] = lds + St::kBytes + 4 * half * St::kRowBytes + 4 * (32 * i + col);
    }
    const auto lds_frag = [](unsigned at) { return *(const __attribute__((address_space(3))) frag_t*)(uintptr_t)at; };
    const auto lds_float = [](unsigned at) { return *(const __attribute__((address_space(3))) float*)(uintptr_t)at; };

    const auto compute = [&](int it, int buf, auto masked, unsigned long long live, bool edge) {
        constexpr bool kMasked = decltype(masked)::value;
        const unsigned off = 2 * buf * St::kBytes;
        f32x16_t s[kSubs];
#pragma unroll
        for (int j = 0; j < kSubs; ++j) s[j] = zero_acc();
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int j = 0; j < kSubs; ++j) mma<T>(s[j], lds_frag((k_base ^ (32 * f)) + off + 32 * j * St::kRowBytes), qf[f]);
        unsigned seen[kSubs];
        if constexpr (kMasked) {
            const int left = lim - it * kKv;                   // rows of this stage that the query sees
            const unsigned long long bits = (left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1) & live;
#pragma unroll
            for (int j = 0; j < kSubs; ++j) {
                seen[j] = (unsigned)(bits >> (32 * j)) >> (4 * half);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[j][r] = (seen[j] >> acc_row(r, 0)) & 1 ? s[j][r] : -INFINITY;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int j = 0; j < kSubs; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[j][r]);
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
        for (int j = 0; j < kSubs; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[j][r] = exp2_fast(__builtin_fmaf(s[j][r], a.scale_log2e, -ref));
                l += s[j][r];
            }
        const auto value_frag = [&](int t, int i) {            // rows 16 t .. 16 t + 15 (16-bit)
            const s16x4_t x = read_transposed(v_base[i] + off + 16 * t * St::kRowBytes);
            const s16x4_t y = read_transposed(v_base[i] + off + (16 * t + 8) * St::kRowBytes);
            return __builtin_bit_cast(frag_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        const auto value_row = [&](int j, int r, int i) { return lds_float(v_base[i] + off + (32 * j + acc_row(r, 0)) * St::kRowBytes); };
        // Where some query does not see a row, the row's value counts 0 times: an infinity or NaN there must not.  Such a stage
        // (hardly ever there) adds values that are finite, and sees by a second product which queries see one that is not.
        bool odd = false;
        if constexpr (kMasked) if (edge) {
            if constexpr (sizeof(T) == 2) {
                typedef short s16x8_t __attribute__((ext_vector_type(8)));
                typedef unsigned short u16x8_t __attribute__((ext_vector_type(8)));
                s16x8_t up = 0;
                u16x8_t down = 0;
#pragma unroll
                for (int t = 0; t < 2 * kSubs; ++t)
#pragma unroll
                    for (int i = 0; i < kOut; ++i) {
                        const frag_t x = value_frag(t, i);
                        up = __builtin_elementwise_max(up, __builtin_bit_cast(s16x8_t, x));
                        down = __builtin_elementwise_max(down, __builtin_bit_cast(u16x8_t, x));
                    }
#pragma unroll
                for (int e = 0; e < 8; ++e) odd |= up[e] >= 0x7f80 || down[e] >= 0xff80;
            } else {
#pragma unroll
                for (int j = 0; j < kSubs; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
#pragma unroll
                        for (int i = 0; i < kOut; ++i) odd |= !(fabsf(value_row(j, r, i)) < INFINITY);
            }
            odd = __any(odd);
        }
        if constexpr (sizeof(T) == 2) {
            frag_t p[2 * kSubs];
#pragma unroll
            for (int t = 0; t < 2 * kSubs; ++t) {
                bf16x8_t x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = (bf16_t)s[t / 2][8 * (t % 2) + e];
                p[t] = __builtin_bit_cast(frag_t, x);
            }
            if (kMasked && odd) {
#pragma unroll 1
                for (int i = 0; i < kOut; ++i) {
                    f32x16_t sum = zero_acc(), count = zero_acc();
#pragma unroll
                    for (int t = 0; t < 2 * kSubs; ++t) {
                        bf16x8_t x = __builtin_bit_cast(bf16x8_t, value_frag(t, i)), not_finite, sees;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool fine = fabsf((float)x[e]) < INFINITY;
                            x[e] = fine ? x[e] : (bf16_t)0.f;
                            not_finite[e] = (bf16_t)(fine ? 0.f : 1.f);
                            sees[e] = (bf16_t)((seen[t / 2] >> acc_row(8 * (t % 2) + e, 0)) & 1 ? 1.f : 0.f);
                        }
                        mma<T>(sum, __builtin_bit_cast(frag_t, x), p[t]);
                        mma<T>(count, __builtin_bit_cast(frag_t, not_finite), __builtin_bit_cast(frag_t, sees));
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum[r] = count[r] > 0.f ? NAN : sum[r];
#pragma unroll
                    for (int n = 0; n < kOut; ++n) if (n == i) o[n] += sum;
                }
            } else {
#pragma unroll
                for (int t = 0; t < 2 * kSubs; ++t)
#pragma unroll
                    for (int i = 0; i < kOut; ++i) mma<T>(o[i], value_frag(t, i), p[t]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
                f32x16_t count = zero_acc();
#pragma unroll
                for (int j = 0; j < kSubs; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float x = value_row(j, r, i);
                        if (kMasked && odd) {
                            const bool fine = fabsf(x) < INFINITY;
                            count = __builtin_amdgcn_mfma_f32_32x32x2f32(fine ? 0.f : 1.f, (seen[j] >> acc_row(r, 0)) & 1 ? 1.f : 0.f, count, 0, 0, 0);
                            x = fine ? x : 0.f;
                        }
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[j][r], o[i], 0, 0, 0);
                    }
                if (kMasked && odd)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[i][r] = count[r] > 0.f ? NAN : o[i][r];
            }
        }
    };

    // Stages come last rows first.  One is in flight while one is worked on; rows of pages are looked up two further on.
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
        unsigned long long live = ~0ull;
        if constexpr (kPaged) {
            live = live_of[it % kHold];
            live = ((unsigned long long)(unsigned)scalar((int)(live >> 32)) << 32) | (unsigned)scalar((int)live);
            if (wave == 0) {
                settle(it - 2 + kHold, far, far_mask);
                far = row_trip(it - 3, entry, far_mask);
                entry = table_trip(it - 4);
            }
        }
        if (r0 < n_rows && it * kKv < lim_max && live) {
            const unsigned long long all = kKv == 64 ? ~0ull : (1ull << kKv) - 1;
            const bool edge = it * kKv + kKv > lim_min;
            if (edge || (kPaged && live != all)) compute(it, buf, std::true_type{}, live, edge);
            else compute(it, buf, std::false_type{}, live, false);
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

// ---- joining

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

// Waves of a block (32 query rows each) and blocks that share a tile's rows of keys and values.
PromptPlan plan_prompt(long long sequences, long long rows, long long all_rows, int kv_heads, long long most)
{
    PromptPlan p{};
    const auto blocks = [&](int waves) {
        const int tile = 32 * waves;
        const long long by_sequence = sequences * ((rows + tile - 1) / tile), together = (all_rows + tile - 1) / tile + sequences;
        return kv_heads * (by_sequence < together ? by_sequence : together);
    };
    p.waves = 8;
    while (p.waves > 1 && blocks(p.waves) < 256) p.waves /= 2;
    p.tiles = blocks(p.waves) / kv_heads;
    p.splits = 1;
    const long long n = blocks(p.waves);
    if (n < 512 && most >= 1024) p.splits = (int)std::min({(512 + n - 1) / n, most / 512, 64ll});
    return p;
}

namespace {
template <typename T, int D, bool kPaged>
hipError_t launch(PromptArgs a, const PromptPlan& plan, hipStream_t st)
{
    a.page_shift = 0;
    while (1 << a.page_shift < a.page_size) ++a.page_shift;
    a.page_magic = kPaged ? (unsigned)(((1ull << (31 + a.page_shift)) + a.page_size - 1) / a.page_size) : 0;
    a.splits = plan.splits;
    const dim3 grid((unsigned)(plan.tiles * a.kv_heads), plan.splits);
    if (plan.waves == 8) prompt_kernel<T, D, kPaged, 8><<<grid, 512, 0, st>>>(a);
    else if (plan.waves == 4) prompt_kernel<T, D, kPaged, 4><<<grid, 256, 0, st>>>(a);
    else if (plan.waves == 2) prompt_kernel<T, D, kPaged, 2><<<grid, 128, 0, st>>>(a);
    else prompt_kernel<T, D, kPaged, 1><<<grid, 64, 0, st>>>(a);
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
