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

// 8 elements of a row as they are; `wide`: the address is a multiple of 16 bytes
template <typename T> struct Piece { frag_t f[8 * sizeof(T) / 16]; };
template <typename T> struct Elems { T x[8]; };

template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* p, bool wide)
{
    Piece<T> r;
    if (wide) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(r) / 16); ++i) r.f[i] = reinterpret_cast<const frag_t*>(p)[i];
    } else {
        Elems<T> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.x[i] = p[i];
        r = __builtin_bit_cast(Piece<T>, e);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void store_piece(T* p, bool wide, const Piece<T>& r)
{
    if (wide) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(r) / 16); ++i) reinterpret_cast<frag_t*>(p)[i] = r.f[i];
    } else {
        const Elems<T> e = __builtin_bit_cast(Elems<T>, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = e.x[i];
    }
}

template <typename T>
__device__ __forceinline__ void unpack8(const Piece<T>& r, float (&x)[8])
{
    const Elems<T> e = __builtin_bit_cast(Elems<T>, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_float(e.x[i]);
}

template <typename T>
__device__ __forceinline__ Piece<T> pack8(const float (&x)[8])
{
    Elems<T> e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.x[i] = (T)x[i];              // round to nearest even
    return __builtin_bit_cast(Piece<T>, e);
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

// A thread takes 16 elements of one row: the two halves of 8 pairs (or 16 elements that only move).  It reads them all
// before it writes any, so queries may be turned in place.
template <typename T, int D>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr int kItems = D / 16;
    const int rows = a.q_heads_used + 2 * a.kv_heads;                          // of one token: queries, keys, values
    const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
    const int item = (int)(idx % kItems);
    const long long rest = idx / kItems;
    const int row = (int)(rest % rows);
    const long long token = rest / rows;
    if (token >= (long long)a.batch * a.n_new) return;
    const int b = (int)(token / a.n_new), i = (int)(token % a.n_new);

    const int n = a.new_len ? min(max(a.new_len[b], 0), a.n_new) : a.n_new;
    const long long capacity = (long long)a.max_pages * a.page_size;
    const long long slot = (long long)a.start[b] + i;
    if (a.len_out && i == 0 && row == 0 && item == 0)
        a.len_out[b] = (int)min(max((long long)a.start[b] + n, 0ll), capacity);
    if (i >= n) return;

    const bool is_q = row < a.q_heads_used, is_k = !is_q && row < a.q_heads_used + a.kv_heads;
    const int head = is_q ? row : is_k ? row - a.q_heads_used : row - a.q_heads_used - a.kv_heads;
    const int kv_head = is_q ? head / a.group : head;

    T* dst;
    long long at = 0;
    bool wide_out = true;
    if (is_q) {
        dst = reinterpret_cast<T*>(a.q_out) + b * a.qo_sb + head * a.qo_sh + i * a.qo_sn;
        wide_out = a.qo_wide;
    } else {
        if (slot < 0 || slot >= capacity) return;
        const int page = a.page_table[(size_t)b * a.max_pages + (int)(slot / a.page_size)];
        if (page < 0 || page >= a.num_pages) return;
        at = ((long long)page * a.kv_heads + head) * a.page_size + slot % a.page_size;
        dst = reinterpret_cast<T*>(is_k ? a.k_pages : a.v_pages) + at * D;
    }
    const T* src = is_q   ? reinterpret_cast<const T*>(a.q) + b * a.q_sb + head * a.q_sh + i * a.q_sn
                   : is_k ? reinterpret_cast<const T*>(a.k) + b * a.k_sb + head * a.k_sh + i * a.k_sn
                          : reinterpret_cast<const T*>(a.v) + b * a.v_sb + head * a.v_sh + i * a.v_sn;
    const bool wide_in = is_q ? a.q_wide : is_k ? a.k_wide : a.v_wide;

    const double pos = a.positions ? (double)a.positions[b * a.pos_sb + kv_head * a.pos_sh + i * a.pos_sn] : (double)slot;
    if (is_k && item == 0 && a.pos_pages) a.pos_pages[at] = (int)pos;

    const bool paired = item < a.rot / 16;
    const bool halves = paired && !a.interleaved;                              // 8 columns of each half, else 16 in a row
    const int e0 = halves ? 8 * item : 16 * item, e1 = halves ? 8 * item + a.rot / 2 : 16 * item + 8;
    Piece<T> p0 = load_piece(src + e0, wide_in), p1 = load_piece(src + e1, wide_in);
    if (paired && (is_q || is_k)) {
        float x[8], y[8], c[8], s[8];
        unpack8(p0, x);
        unpack8(p1, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(pos, a.inv_freq[8 * item + e], c[e], s[e]);
        if (halves) {
#pragma unroll
            for (int e = 0; e < 8; ++e) rotate(x[e], y[e], c[e], s[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                rotate(x[2 * e], x[2 * e + 1], c[e], s[e]);
                rotate(y[2 * e], y[2 * e + 1], c[e + 4], s[e + 4]);
            }
        }
        p0 = pack8<T>(x);
        p1 = pack8<T>(y);
    }
    store_piece(dst + e0, wide_out, p0);
    store_piece(dst + e1, wide_out, p1);
}

hipError_t launch_append(const AppendArgs& a, int head_dim, bool f32, hipStream_t st)
{
    const long long threads = (long long)a.batch * a.n_new * (a.q_heads_used + 2 * a.kv_heads) * (head_dim / 16);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (f32) {
        if (head_dim == 64) append_kernel<float, 64><<<grid, 256, 0, st>>>(a);
        else append_kernel<float, 128><<<grid, 256, 0, st>>>(a);
    } else {
        if (head_dim == 64) append_kernel<bf16_t, 64><<<grid, 256, 0, st>>>(a);
        else append_kernel<bf16_t, 128><<<grid, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace ems
