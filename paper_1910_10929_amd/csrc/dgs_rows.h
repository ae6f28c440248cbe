// Helpers of the training-block kernels: eight consecutive values of a row in a lane, element types, row sums, and the
// codes of a checkpoint.
//
// A lane holds values c .. c + 7 of a row, c a multiple of 8, so that the four lanes of a quad hold the 32 columns that
// share an exponent, and a run's largest magnitude is two quad permutes away.  Loads and stores are 16 bytes (8 for codes)
// at any alignment of the element type; the last, shorter piece of a row is loaded as the row's last eight values and put in
// place (element by element where a row has fewer than eight), and stored element by element.
#pragma once
#include "dgs_wave.h"
#include "../../include/dgs_blocks.h"

namespace dgs {

typedef _Float16 f16;
#ifdef DGS_HOST_EMULATION
struct bf16 { uint16_t bits; };
#else
typedef __bf16 bf16;
#endif

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(f16 v) { return (float)v; }
#ifdef DGS_HOST_EMULATION
__device__ __forceinline__ float to_float(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
#else
__device__ __forceinline__ float to_float(bf16 v) { return (float)v; }
#endif

template <class T> __device__ __forceinline__ T from_float(float v) { return (T)v; }
#ifdef DGS_HOST_EMULATION
template <> inline bf16 from_float<bf16>(float v)      // to nearest, halfway cases to even
{
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return bf16{(uint16_t)((u >> 16) | 0x40u)};
    return bf16{(uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16)};
}
#endif

// The same number, of which the compiler knows nothing: an address stays a row's pointer in scalar registers plus this
// offset, where it would otherwise keep a 64-bit pointer a lane for every matrix of a loop.
__device__ __forceinline__ uint32_t opaque(uint32_t v)
{
#ifndef DGS_HOST_EMULATION
    asm volatile("" : "+v"(v));
#endif
    return v;
}

// ---------------------------------------------------------------------------
// eight values of a row
// ---------------------------------------------------------------------------

// What is loaded, before it is unpacked (so that loads can be issued a row ahead at the registers the memory format takes).
template <class T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };

// `n` (at most 8) values at p; the others are 0.
template <class T> __device__ __forceinline__ Raw8<T> load8(const T *p, uint32_t n)
{
    Raw8<T> r;
    if (n >= 8) {
        const u32x4_any *q = (const u32x4_any *)p;
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
            const u32x4_any v = q[i];
            r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
        }
    } else {
        T t[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) t[i] = i < n ? p[i] : from_float<T>(0.0f);
        __builtin_memcpy(&r, t, sizeof(r));
    }
    return r;
}

template <class T> __device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&v)[8])
{
    T t[8];
    __builtin_memcpy(t, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
}
template <> __device__ __forceinline__ void unpack8<bf16>(const Raw8<bf16> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
    }
}

// Matrices are stored past the caches' replacement order (non-temporal): 16384 x 4096 bfloat16 edges with their checkpoints
// and the decoding of those 222 us against 238, 151 M values encoded and decoded 222 against 243, and 8192 x 768 edges, which the
// caches would hold, 38 against 41.  (Non-temporal loads cost the small ones a fifth.)
template <class T> __device__ __forceinline__ void store8(T *row, uint32_t c, uint32_t n, const float (&v)[8])
{
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_float<T>(v[i]);
    T *const p = (T *)((char *)row + opaque(c * (uint32_t)sizeof(T)));
    if (n == 8) {
        Raw8<T> r;
        __builtin_memcpy(&r, t, sizeof(r));
        u32x4_any *q = (u32x4_any *)p;
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
            u32x4_any o;
            o.x = r.w[4 * i]; o.y = r.w[4 * i + 1]; o.z = r.w[4 * i + 2]; o.w = r.w[4 * i + 3];
            __builtin_nontemporal_store(o, q + i);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i)
            if (i < n) p[i] = t[i];
    }
}

// The same for a type that is known at run time: a vector of parameters, a gate.
__device__ __forceinline__ void load8_f32(const float *p, uint32_t n, float (&v)[8]) { unpack8(load8(p, n), v); }

// ---------------------------------------------------------------------------
// eight values of a row, loaded without a branch
// ---------------------------------------------------------------------------
// A load inside a branch makes the compiler wait for everything in flight where the branch ends.  So every lane loads eight
// values that exist: the last eight of the row where its own eight end beyond it, moved into place afterwards.  Lanes that
// hold no column at all load those too, and are left out of sums and stores.  Rows of fewer than eight columns (TINY) are
// loaded element by element.
struct Place8 { uint32_t c, at, n; };       // first column, first column loaded, columns that exist

template <bool TINY> __device__ __forceinline__ Place8 place8(uint32_t c, uint32_t cols)
{
    Place8 p;
    p.c = c;
    p.n = c >= cols ? 0u : min(8u, cols - c);
    p.at = TINY ? 0u : min(c, cols - 8u);
    return p;
}

template <bool TINY, class T> __device__ __forceinline__ Raw8<T> load_at(const T *row, uint32_t at, uint32_t cols)
{
    Raw8<T> r;
    if constexpr (TINY) {
        T t[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) t[i] = row[min(i, cols - 1u)];
        __builtin_memcpy(&r, t, sizeof(r));
    } else {
        const u32x4_any *q = (const u32x4_any *)((const char *)row + opaque(at * (uint32_t)sizeof(T)));
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
            const u32x4_any v = q[i];
            r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
        }
    }
    return r;
}

// The words of w moved down by `by` (fewer than 8) elements of 1, 2 or 4 bytes; 0 comes in behind.
template <uint32_t WORDS, uint32_t BYTES> __device__ __forceinline__ void move_down(uint32_t (&w)[WORDS], uint32_t by)
{
#pragma unroll
    for (uint32_t step = 4; step >= 1; step /= 2) {
        const uint32_t bits = step * BYTES * 8;
        const bool move = (by & step) != 0;
#pragma unroll
        for (uint32_t i = 0; i < WORDS; ++i) {
            uint32_t v;
            if (bits >= 32) {
                v = i + bits / 32 < WORDS ? w[i + bits / 32 < WORDS ? i + bits / 32 : 0] : 0u;
            } else {
                const uint32_t up = i + 1 < WORDS ? w[i + 1 < WORDS ? i + 1 : 0] : 0u;
                v = (w[i] >> (bits & 31u)) | (up << ((32u - bits) & 31u));
            }
            w[i] = move ? v : w[i];
        }
    }
}

// What was loaded, in place, 0 where there is no column.  Lanes without columns are left as they are.  Only rows whose length
// is no multiple of eight need this.
template <bool TINY, class T> __device__ __forceinline__ void in_place(Raw8<T> &r, const Place8 &p)
{
    if constexpr (TINY) {
        T t[8];
        __builtin_memcpy(t, &r, sizeof(r));
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) t[i] = i < p.n ? t[i] : from_float<T>(0.0f);
        __builtin_memcpy(&r, t, sizeof(r));
    } else {
        move_down<sizeof(r.w) / 4, sizeof(T)>(r.w, p.n ? p.c - p.at : 0u);
    }
}

// How many of the eight values from column c on exist.
__device__ __forceinline__ uint32_t live8(uint32_t c, uint32_t cols) { return c >= cols ? 0u : min(8u, cols - c); }

// ---------------------------------------------------------------------------
// sums over lanes
// ---------------------------------------------------------------------------

#ifdef DGS_HOST_EMULATION
__device__ __forceinline__ uint32_t lane_read(uint32_t v, uint32_t lane) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(lane * 4), (int)v); }
__device__ __forceinline__ uint32_t quad_xor1(uint32_t v) { return lane_read(v, lane_id() ^ 1u); }
__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) { return lane_read(v, lane_id() ^ 2u); }
__device__ __forceinline__ uint32_t half_mirror(uint32_t v) { return lane_read(v, lane_id() ^ 7u); }
__device__ __forceinline__ uint32_t row_mirror(uint32_t v) { return lane_read(v, lane_id() ^ 15u); }
#else
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t quad_xor1(uint32_t v) { return dpp<0xB1>(v); }      // quad_perm 1 0 3 2
__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) { return dpp<0x4E>(v); }      // quad_perm 2 3 0 1
__device__ __forceinline__ uint32_t half_mirror(uint32_t v) { return dpp<0x141>(v); }
__device__ __forceinline__ uint32_t row_mirror(uint32_t v) { return dpp<0x140>(v); }
#endif

// The sum over the wavefront, the same bits in every lane: within rows of 16 lanes by lane permutes, then the four rows.
__device__ __forceinline__ float wave_sum(float v)
{
    v += __uint_as_float(quad_xor1(__float_as_uint(v)));
    v += __uint_as_float(quad_xor2(__float_as_uint(v)));
    v += __uint_as_float(half_mirror(__float_as_uint(v)));
    v += __uint_as_float(row_mirror(__float_as_uint(v)));
    const int b = (int)__float_as_uint(v);
    const float r0 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 0));
    const float r1 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 16));
    const float r2 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 32));
    const float r3 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 48));
    return (r0 + r1) + (r2 + r3);
}

// Sums over a team of WAVES wavefronts, of which a workgroup holds ALL / WAVES; with more than one wavefront to a team, every
// thread of the workgroup calls this the same number of times.  Successive calls use the two halves of `lds` in turn (`turn`
// flips), which makes one barrier a call enough: whoever writes a half again has passed the barrier of the other half's call,
// and with it every reader of the first.
template <int ALL> struct TeamLds { float v[2][2][ALL]; };

template <int WAVES, int ALL, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], TeamLds<ALL> &lds, uint32_t &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        float (*half)[ALL] = lds.v[turn];
        turn ^= 1u;
        const uint32_t wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
        if (lane_id() == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) half[i][wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = half[i][first];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += half[i][first + w];
            v[i] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// checkpoint codes
// ---------------------------------------------------------------------------

// The exponent byte of the run that this quad of lanes holds, from the bits of its largest magnitude: with top = m 2^E, m in
// [1, 2), the exponent is E - 6 where 64 m < 127.5, one more otherwise (a carry out of the mantissa).
__device__ __forceinline__ uint32_t run_byte(const float (&v)[8], bool any)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = any ? top : 0u;
    top = max(top, quad_xor1(top));
    top = max(top, quad_xor2(top));
    const int byte = (int)((top + 0x10000u) >> 23) - 6;
    return top >= 0x7F800000u ? 255u : (uint32_t)min(max(byte, 1), 248);
}

// Eight codes of the run with exponent byte `byte`.  v 2^-e + 1.5 2^23 in one rounding leaves the nearest whole number
// (halfway cases to even) in the low mantissa bits, its low byte being the code.
__device__ __forceinline__ void encode8(const float (&v)[8], uint32_t byte, uint32_t (&q)[2])
{
    const float scale = __uint_as_float((254u - byte) << 23);
    uint32_t b[8];
    if (byte < 248u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__builtin_fmaf(v[i], scale, 12582912.0f)) & 0xFFu;
    } else {      // the largest exponent, where 128 is cut to 127; or nothing finite
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = min(max(v[i] * scale, -127.0f), 127.0f);
            b[i] = byte == 255u ? 0u : __float_as_uint(c + 12582912.0f) & 0xFFu;
        }
    }
    q[0] = b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
    q[1] = b[4] | (b[5] << 8) | (b[6] << 16) | (b[7] << 24);
}

__device__ __forceinline__ float run_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23); }

__device__ __forceinline__ void decode8(const uint32_t (&q)[2], float scale, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * scale;
}

template <bool TINY> __device__ __forceinline__ void load_codes_at(const int8_t *row, uint32_t at, uint32_t cols, uint32_t (&q)[2])
{
    if constexpr (TINY) {
        q[0] = q[1] = 0;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) q[i >> 2] |= (uint32_t)(uint8_t)row[min(i, cols - 1u)] << (8 * (i & 3));
    } else {
        const u32x2_any v = *(const u32x2_any *)(row + opaque(at));
        q[0] = v.x;
        q[1] = v.y;
    }
}
template <bool TINY> __device__ __forceinline__ void codes_in_place(uint32_t (&q)[2], const Place8 &p)
{
    if constexpr (TINY) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i >= p.n) q[i >> 2] &= ~(0xFFu << (8 * (i & 3)));
    } else {
        move_down<2, 1>(q, p.n ? p.c - p.at : 0u);
    }
}

// `n` codes at p; the others are 0.
__device__ __forceinline__ void load_codes(const int8_t *p, uint32_t n, uint32_t (&q)[2])
{
    if (n >= 8) {
        const u32x2_any v = *(const u32x2_any *)p;
        q[0] = v.x;
        q[1] = v.y;
    } else {
        q[0] = q[1] = 0;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) q[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    }
}
__device__ __forceinline__ void store_codes(int8_t *row, uint32_t c, uint32_t n, const uint32_t (&q)[2])
{
    int8_t *const p = row + opaque(c);
    if (n == 8) {
        u32x2_any v;
        v.x = q[0];
        v.y = q[1];
        __builtin_nontemporal_store(v, (u32x2_any *)p);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i)
            if (i < n) p[i] = (int8_t)(q[i >> 2] >> (8 * (i & 3)));
    }
}

// Values c .. c + 7 of a row as a checkpoint: every lane of the wavefront calls this (n = 0 where the row has ended).
// Values beyond the row are 0 in v, or there are none of the row (n = 0).
__device__ __forceinline__ void save8(int8_t *row, uint8_t *exps, uint32_t c, uint32_t n, const float (&v)[8])
{
    const uint32_t byte = run_byte(v, n != 0);
    if (n == 0) return;
    uint32_t q[2];
    encode8(v, byte, q);
    store_codes(row, c, n, q);
    if ((c & (DGS_CHECKPOINT_RUN - 1)) == 0) exps[opaque(c / DGS_CHECKPOINT_RUN)] = (uint8_t)byte;
}

// ---------------------------------------------------------------------------
// host side: arguments
// ---------------------------------------------------------------------------

static inline uint64_t type_bytes(int type) { return type == DGS_F32 ? 4u : 2u; }
static inline bool is_type(int type) { return type >= DGS_F32 && type <= DGS_BF16; }
static inline bool aligned_to(const void *p, uint64_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
static inline bool matrix_ok(const void *p, uint64_t stride, uint64_t cols, int type)
{
    return p && stride >= cols && stride < (1ull << 32) && aligned_to(p, type_bytes(type));
}
static inline bool codes_ok(const dgs_codes &c, uint64_t cols)
{
    return c.codes && c.exps && c.codes_stride >= cols && c.codes_stride < (1ull << 32)
        && c.exps_stride >= (cols + DGS_CHECKPOINT_RUN - 1) / DGS_CHECKPOINT_RUN && c.exps_stride < (1ull << 32);
}
// What a launch that was enqueued without an event leaves.
static inline int launched() { return hipGetLastError() == hipSuccess ? DGS_OK : DGS_EHIP; }

}  // namespace dgs
