// Appending keys and values to a paged cache, with the position rotation on the way.
//
// A pair (x1, x2) of frequency f at position t becomes (x1 cos a - x2 sin a, x2 cos a + x1 sin a), a = t f.  The angle is
// formed in 64 bits and cut to an eighth of a turn either way before it is rounded to 32: at t = 10^6 a 32-bit product
// alone is 0.06 radians off.
#include "ems_common.h"
#include "ems_kernels.h"
#include "ems_rows.h"

namespace ems {

namespace {

// 16 bytes of a row as they are; `wide`: the address is a multiple of 16 bytes; kPast: past the caches (nontemporal)
template <typename T> struct Elems { T x[16 / sizeof(T)]; };

template <typename T, bool kPast>
__device__ __forceinline__ frag_t load_piece(const T* p, bool wide)
{
    if (wide) {
        const frag_t* at = reinterpret_cast<const frag_t*>(p);
        return kPast ? __builtin_nontemporal_load(at) : *at;
    }
    Elems<T> e;
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e.x[i] = p[i];
    return __builtin_bit_cast(frag_t, e);
}

template <typename T, bool kPast>
__device__ __forceinline__ void store_piece(T* p, bool wide, const frag_t& f)
{
    if (wide) {
        frag_t* at = reinterpret_cast<frag_t*>(p);
        if constexpr (kPast) __builtin_nontemporal_store(f, at);
        else *at = f;
    } else {
        const Elems<T> e = __builtin_bit_cast(Elems<T>, f);
#pragma unroll
        for (int i = 0; i < (int)(16 / sizeof(T)); ++i) p[i] = e.x[i];
    }
}

// cos and sin of t f
__device__ __forceinline__ void turn(double t, float f, float& c, float& s)
{
    const double turns = t * (double)f * 0.15915494309189533577;       // of a full circle
    const double quarter = __builtin_rint(4.0 * turns);
    const float rest = (float)(4.0 * turns - quarter);                         // quarters, at most half of one
    float cr, sr;
    sincospif(0.5f * rest, &sr, &cr);
    const int n = (int)(quarter - 4.0 * __builtin_floor(0.25 * quarter));      // 0..3
    c = n == 0 ? cr : n == 1 ? -sr : n == 2 ? -cr : sr;
    s = n == 0 ? sr : n == 1 ? cr : n == 2 ? -sr : -cr;
}

__device__ __forceinline__ void rotate(float& u, float& w, float c, float s)
{
    const float x = u;
    u = x * c - w * s;
    w = w * c + x * s;
}

}  // namespace

// A block takes some tokens and the rows (queries, keys, values) of some kv-heads.  Its angles are formed once, a value a
// thread, and shared through LDS: 64-bit products and a sine for every element of every head would be the kernel's time
// (four prompts of 8192 tokens, 40 heads to rotate: 187 us, and 168 so).  Then a lane group takes a row, a lane two pieces
// of 16 bytes that hold both halves of its pairs, kAhead rows requested together; a lane reads all of its elements before it
// writes any, so queries may be turned in place.  Memory bounds it: those prompts, 805 MB read and written, 156 us, 5.2 TB/s.
template <typename T, int D, bool kPast>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr int kPer = 16 / (int)sizeof(T);                  // elements of a piece: a lane takes two pieces of a row
    constexpr int kItems = D / (2 * kPer), kGroups = 256 / kItems, kAhead = 4;
    __shared__ __align__(16) float cs[kGroups][2][D / 2];
    const int n_tok = a.tokens;                                // of a block: a power of two
    const int h0 = blockIdx.y * a.heads, heads = min(a.heads, a.kv_heads - h0);       // its kv-heads
    const int tok0 = blockIdx.x * n_tok, all = a.batch * a.n_new;
    const auto place = [&](int token, int& b, int& i) { b = token / a.n_new; i = token - b * a.n_new; };
    const auto position = [&](int b, int i) -> double {
        if (a.positions) return a.positions[b * a.pos_sb + h0 * a.pos_sh + i * a.pos_sn];       // (one head where each has its own)
        return (double)a.start[b] + i;
    };
    const int half = a.rot / 2;
    for (int x = threadIdx.x; x < n_tok * half; x += 256) {
        const int t = x / half, e = x - t * half;
        int b, i;
        place(min(tok0 + t, all - 1), b, i);
        turn(position(b, i), a.inv_freq[e], cs[t][0][e], cs[t][1][e]);
    }
    __syncthreads();

    const int item = threadIdx.x % kItems, group = threadIdx.x / kItems, t = group % n_tok;
    if (tok0 + t >= all) return;
    int b, i;
    place(tok0 + t, b, i);
    const int n = a.new_len ? min(max(a.new_len[b], 0), a.n_new) : a.n_new;
    const long long capacity = (long long)a.max_pages * a.page_size;
    const long long slot = (long long)a.start[b] + i;
    if (a.len_out && i == 0 && h0 == 0 && group < n_tok && item == 0)
        a.len_out[b] = (int)min(max((long long)a.start[b] + n, 0ll), capacity);
    if (i >= n) return;

    // the token's row in the cache, of kv-head 0; none: only its queries are turned
    long long at = -1;
    if (slot >= 0 && slot < capacity) {
        const int page = a.page_table[(size_t)b * a.max_pages + (int)slot / a.page_size];
        if (page >= 0 && page < a.num_pages) at = (long long)page * a.kv_heads * a.page_size + (int)slot % a.page_size;
    }
    // Neighbouring lanes take neighbouring pieces: of the two halves of the rotated columns (paired across the halves, or
    // within each piece), of the two halves of those behind them, and of a row that only moves.
    const int n_paired = a.rot / (2 * kPer);
    const bool paired = item < n_paired;
    const int e0 = paired ? kPer * item : a.rot + kPer * (item - n_paired), e1 = e0 + (paired ? half : (D - a.rot) / 2);
    const int m0 = kPer * item, m1 = m0 + D / 2;
    float c[kPer], s[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int f = !a.interleaved ? kPer * item + e : kPer / 2 * item + e % (kPer / 2) + (e < kPer / 2 ? 0 : half / 2);
        c[e] = paired ? cs[t][0][f] : 1.f;
        s[e] = paired ? cs[t][1][f] : 0.f;
    }

    const int n_q = a.q ? heads * a.group : 0, rows = n_q + 2 * heads;
    const T* q_in = reinterpret_cast<const T*>(a.q) + b * a.q_sb + (long long)h0 * a.group * a.q_sh + i * a.q_sn;
    T* q_out = reinterpret_cast<T*>(a.q_out) + b * a.qo_sb + (long long)h0 * a.group * a.qo_sh + i * a.qo_sn;
    const T* k_in = reinterpret_cast<const T*>(a.k) + b * a.k_sb + h0 * a.k_sh + i * a.k_sn;
    const T* v_in = reinterpret_cast<const T*>(a.v) + b * a.v_sb + h0 * a.v_sh + i * a.v_sn;
    const int step = kGroups / n_tok;
    for (int r0 = group / n_tok; r0 < rows; r0 += kAhead * step) {
        frag_t p0[kAhead], p1[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + u * step, k = r - n_q, v = k - heads;
            if (r >= rows || (r >= n_q && at < 0)) continue;
            const T* src = r < n_q ? q_in + r * a.q_sh : v < 0 ? k_in + k * a.k_sh : v_in + v * a.v_sh;
            const bool wide = r < n_q ? a.q_wide : v < 0 ? a.k_wide : a.v_wide;
            p0[u] = load_piece<T, kPast>(src + (v < 0 ? e0 : m0), wide);
            p1[u] = load_piece<T, kPast>(src + (v < 0 ? e1 : m1), wide);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + u * step, k = r - n_q, v = k - heads;
            if (r >= rows || (r >= n_q && at < 0)) continue;
            if (paired && v < 0) {
                float x[kPer], y[kPer];
                Pack<T>::unpack(p0[u], x);
                Pack<T>::unpack(p1[u], y);
                if (!a.interleaved) {
#pragma unroll
                    for (int e = 0; e < kPer; ++e) rotate(x[e], y[e], c[e], s[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < kPer / 2; ++e) {
                        rotate(x[2 * e], x[2 * e + 1], c[e], s[e]);
                        rotate(y[2 * e], y[2 * e + 1], c[kPer / 2 + e], s[kPer / 2 + e]);
                    }
                }
                p0[u] = Pack<T>::pack(x);
                p1[u] = Pack<T>::pack(y);
            }
            const long long row = at + (long long)(h0 + (v < 0 ? k : v)) * a.page_size;
            T* dst = r < n_q ? q_out + r * a.qo_sh : reinterpret_cast<T*>(v < 0 ? a.k_pages : a.v_pages) + row * D;
            const bool wide = r >= n_q || a.qo_wide;
            store_piece<T, kPast>(dst + (v < 0 ? e0 : m0), wide, p0[u]);
            store_piece<T, kPast>(dst + (v < 0 ? e1 : m1), wide, p1[u]);
            if (a.pos_pages && r >= n_q && v < 0 && item == 0)
                a.pos_pages[row] = a.positions ? a.positions[b * a.pos_sb + (h0 + k) * a.pos_sh + i * a.pos_sn] : (int)slot;
        }
    }
}

// Tokens of a block: eight rows for a lane group if there are that few (four prompts of 8192 tokens of 48 rows by 16 tokens a
// block, where eight give it 12 rows: 182 us, by 8: 168).
int append_tokens(int rows, int row_bytes)
{
    const int groups = 256 / (row_bytes / 32);
    int n = 1;
    while (n < groups && n * rows < 8 * groups) n *= 2;
    return n;
}

namespace {
template <typename T, int D>
hipError_t launch(AppendArgs a, hipStream_t st)
{
    const long long all = (long long)a.batch * a.n_new;
    const int rows = (a.q ? a.kv_heads * a.group : 0) + 2 * a.kv_heads;
    // What the last-level cache (256 MB) cannot hold goes past it: four prompts of 8192 tokens (805 MB) take 156 us instead
    // of 168, 100 MB 38 instead of 23, whose pages stay for the attention that reads them.  (Between them nothing was compared; 149 MB
    // take 44 us, staying.)
    const bool past = 2ll * D * (long long)sizeof(T) * all * rows > 256ll << 20;
    // Tokens and kv-heads of a block: all heads, and tokens for eight rows a lane group; less, heads first, until there are
    // two blocks a compute unit.  Where heads have positions of their own and there is a rotation, a block has one.
    a.tokens = append_tokens(rows, D * (int)sizeof(T));
    a.heads = a.pos_sh != 0 && a.rot ? 1 : a.kv_heads;
    const auto blocks = [&] { return (all + a.tokens - 1) / a.tokens * ((a.kv_heads + a.heads - 1) / a.heads); };
    while (a.heads > 1 && blocks() < 512) a.heads = (a.heads + 1) / 2;
    while (a.tokens > 1 && blocks() < 512) a.tokens /= 2;
    const dim3 grid((unsigned)((all + a.tokens - 1) / a.tokens), (a.kv_heads + a.heads - 1) / a.heads);
    if (past) append_kernel<T, D, true><<<grid, 256, 0, st>>>(a);
    else append_kernel<T, D, false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_append(const AppendArgs& a, int head_dim, bool f32, hipStream_t st)
{
    if (f32) return head_dim == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
    return head_dim == 64 ? launch<bf16_t, 64>(a, st) : launch<bf16_t, 128>(a, st);
}

}  // namespace ems
