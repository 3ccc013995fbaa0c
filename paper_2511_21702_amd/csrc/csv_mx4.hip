// 4-bit microscaled rows and the product with a head of such rows.
//
//   quantize_kernel     blocks of 32 elements -> one scale byte and 32 four-bit codes, row-major or in matrix-core tiles
//   dequantize_kernel   the values that row-major codes stand for
//   lay_out_kernel      row-major codes of a head -> tiles
//   product_kernel, many_kernel   out[b, i] = <W_i, h_b> + b_i on the matrix cores
//
// A tile is 16 rows x 128 elements: lane l of a wave holds the 32 elements of block l / 16 of row l % 16 (16 bytes) and that
// block's scale, which is how v_mfma_scale_f32_16x16x128_f8f6f4 takes an operand.  Codes of a tile are 1 KB in lane order; the
// scales of four tiles that follow each other along the row are one dword per lane, byte c for tile c.
// A head is cut into bands of 64 rows.  A band is one piece of memory in the order in which it is read: for every four steps of 128
// elements the scales of its four tiles (1 KB), then for each step the codes of its four tiles (4 KB).  Bands are no power of two apart,
// so that blocks that start together do not ask for the same memory channels.
//
// Times here and below are those of a pass among others.  A head of 279 MB (128256 x 4096) that is read again and again finds part of itself in the
// last-level cache; where heads change from pass to pass, the figure is called a fresh head's.
#include "csv_common.h"

#include <stdlib.h>
#include <type_traits>

#define BLK 32        // elements of a block
#define CHUNK 128     // elements of a row in a tile; rows are padded to a multiple of it
#define HEAD_ROWS 256 // rows of a head are padded to a multiple of it (with codes 0), so that no product kernel tests a row before it stores

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

struct csv_mx4_head {
    int V, d, device;
    int chunks;         // tiles along a row
    uint8_t* bands;     // [rows / 64][band_bytes(chunks)]
    float* bias;        // [V] or NULL
};

static inline int chunks_of(int d) { return (d + CHUNK - 1) / CHUNK; }
__host__ __device__ static inline int64_t band_bytes(int chunks) { return (int64_t)((chunks + 3) >> 2) * 1024 + (int64_t)chunks * 4096; }
// bytes from the start of a band to the scales of steps 4q .. 4q + 3, and to the codes of step c
__host__ __device__ static inline int64_t scales_at(int q) { return (int64_t)q * (1024 + 4 * 4096); }
__host__ __device__ static inline int64_t codes_at(int c) { return (int64_t)c * 4096 + ((c >> 2) + 1) * 1024; }

// ------------------------------------------------------------------------------------------------ rounding
// Eight elements of a lane; four lanes hold a block.  The scale is taken from the exponent field of the largest magnitude alone:
// floor(log2) of a normal float32 is its field - 127, and every subnormal is below the smallest scale anyway.
// x * 2^-e is exact (a result below float32's range rounds to 0 either way), so the one rounding is the conversion's, to nearest even.
struct Elems8 {
    float v[8];
};
__device__ __forceinline__ Elems8 widen8(const v4u& u) {
    return {{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y), bf16_lo(u.z), bf16_hi(u.z), bf16_lo(u.w), bf16_hi(u.w)}};
}
__device__ __forceinline__ Elems8 load8(const uint16_t* p) { return widen8(*(const v4u*)p); }
__device__ __forceinline__ Elems8 load8(const float* p) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ uint32_t scale_of(uint32_t largest) {    // from the float32 pattern of the largest magnitude
    const uint32_t field = largest >> 23;
    return field == 255u ? 255u : field > 2u ? field - 2u : 0u;
}
__device__ __forceinline__ uint32_t codes8(const Elems8& x, uint32_t scale) {
    const float inv = __uint_as_float((254u - (scale == 255u ? 0u : scale)) << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[0] * inv, x.v[1] * inv, 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[2] * inv, x.v[3] * inv, 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[4] * inv, x.v[5] * inv, 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[6] * inv, x.v[7] * inv, 1.0f, 3);
    return scale == 255u ? 0u : r;
}
__device__ __forceinline__ uint32_t largest8(const Elems8& x, uint32_t m) {
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x.v[j]) & 0x7fffffffu);
    return m;
}
__device__ __forceinline__ uint32_t round8(const Elems8& x, uint32_t& scale) {
    uint32_t m = largest8(x, 0);
    m = max(m, (uint32_t)dpp_move<0xB1, 0xf>((int)m, (int)m));   // quad_perm [1,0,3,2]
    m = max(m, (uint32_t)dpp_move<0x4E, 0xf>((int)m, (int)m));   // quad_perm [2,3,0,1]
    scale = scale_of(m);
    return codes8(x, scale);
}

// One wave: 512 elements of a row (blockIdx.x), rows blockIdx.y * 4 + wave and every 4 * gridDim.y rows further.  TILES: codes and scales go
// to tiles; rows past `rows` (up to rows_out) are zeros.  Bound by memory: four lanes share a block, so that every load and store of a wave is
// one piece (128256 x 4096 bf16: 226 us, 5.9 TB/s read and written).
template <typename T, bool TILES>
__global__ __launch_bounds__(256) void quantize_kernel(const T* __restrict__ x, int64_t ld, int rows, int rows_out, int d, int chunks,
                                                        uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const int lane = threadIdx.x & 63, e0 = blockIdx.x * 512 + lane * 8, dp = chunks * CHUNK;
    if (e0 >= dp) return;                                        // whole quads leave: dp is a multiple of 128
    for (int row = blockIdx.y * 4 + (threadIdx.x >> 6); row < rows_out; row += 4 * gridDim.y) {
        Elems8 v = {};
        if (row < rows && e0 < d) v = load8(x + (int64_t)row * ld + e0);
        uint32_t s;
        const uint32_t c = round8(v, s);
        if (TILES) {
            const int tile = row >> 4, chunk = e0 >> 7, blk = (e0 >> 5) & 3, l = blk * 16 + (row & 15);
            *(uint32_t*)(codes + ((int64_t)tile * chunks + chunk) * 1024 + l * 16 + ((e0 >> 1) & 15)) = c;
            if ((lane & 3) == 0) scales[(((int64_t)tile * ((chunks + 3) >> 2) + (chunk >> 2)) * 64 + l) * 4 + (chunk & 3)] = (uint8_t)s;
        } else {
            *(uint32_t*)(codes + (int64_t)row * (dp >> 1) + (e0 >> 1)) = c;
            if ((lane & 3) == 0) scales[(int64_t)row * (dp >> 5) + (e0 >> 5)] = (uint8_t)s;
        }
    }
}

// One wave: 512 elements of a row, 16 bytes of values per lane and store, side by side.  They leave past the caches: four times what came in, and
// read by another kernel at the earliest (128256 x 4096 to bf16 235 -> 225 us; 237 alone under a profiler).
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int d, int chunks,
                                                          T* __restrict__ x, int64_t ld) {
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, dp = chunks * CHUNK;
    for (int row = blockIdx.y * 4 + (threadIdx.x >> 6); row < rows; row += 4 * gridDim.y) {
#pragma unroll
        for (int e0 = blockIdx.x * 512 + lane * E, n = 0; n < 512 / (64 * E); ++n, e0 += 64 * E) {
            if (e0 >= d) continue;
            const uint8_t* from = codes + (int64_t)row * (dp >> 1) + (e0 >> 1);
            const float s = __uint_as_float((uint32_t)scales[(int64_t)row * (dp >> 5) + (e0 >> 5)] << 23);   // exponent field 0: 2^-127; 255: NaN
            const uint32_t c = E == 8 ? *(const uint32_t*)from : *(const uint16_t*)from;
            const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
            if constexpr (E == 4) __builtin_nontemporal_store(v4f{a[0], a[1], b[0], b[1]}, (v4f*)(x + (int64_t)row * ld + e0));
            else {
                // the values have two significant bits: the high half of the float32 pattern is the bfloat16
                const v2f e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
                auto both = [](const v2f& v) { return (__float_as_uint(v[0]) >> 16) | (__float_as_uint(v[1]) & 0xffff0000u); };
                __builtin_nontemporal_store(v4u{both(a), both(b), both(e), both(f)}, (v4u*)(x + (int64_t)row * ld + e0));
            }
        }
    }
}

// One thread: 16 bytes of a tile, and at the first of four steps a dword of scales.  What the padding of a row holds is not taken over.
__global__ __launch_bounds__(256) void lay_out_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int V, int d, int chunks, int64_t pieces,
                                                       uint8_t* __restrict__ bands) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int l = (int)(i & 63), g = l >> 4, tile = (int)(i >> 6) & 3;
    const int64_t t = i >> 8;
    const int chunk = (int)(t % chunks);
    const int64_t band = t / chunks, row = band * 64 + tile * 16 + (l & 15);
    uint8_t* to = bands + band * band_bytes(chunks);
    uint4 c = make_uint4(0, 0, 0, 0);
    const int left = d - chunk * CHUNK - g * BLK;      // elements of the row from this block on, a multiple of 8
    if (row < V && left > 0) {
        c = *(const uint4*)(codes + row * chunks * 64 + chunk * 64 + g * 16);
        if (left <= 24) c.w = 0;
        if (left <= 16) c.z = 0;
        if (left <= 8) c.y = 0;
    }
    *(uint4*)(to + codes_at(chunk) + tile * 1024 + l * 16) = c;
    if ((chunk & 3) == 0) {
        uint32_t s = 0;
        for (int k = 0; k < 4; ++k)
            if (row < V && left > k * CHUNK) s |= (uint32_t)scales[(row * chunks + chunk + k) * 4 + g] << (8 * k);
        *(uint32_t*)(to + scales_at(chunk >> 2) + tile * 256 + l * 4) = s;
    }
}

// ------------------------------------------------------------------------------------------------ product
struct LogitsArgs {
    const uint8_t* bands;
    const float* bias;
    int V, d, chunks, B;
    int blocks;                 // blocks of rows
    int groups;                 // blocks of hidden states
    const uint16_t* h;          // bf16 [B, d]
    const uint8_t* hc;          // or 4-bit tiles of it
    const uint32_t* hs;
    void* out;
    int lines;                  // rows of the output start at multiples of 64 bytes and are as long
};

__device__ __forceinline__ v8i widen(const v4u& u) { return v8i{(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0}; }
__device__ __forceinline__ v8bf bf16_of_fp4(uint32_t c, float s) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1),
               e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2), f = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
    return v8bf{a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]};
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

// Waits for the wave's LDS traffic only: requests to global memory stay in flight across the barrier.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The bias of a block's ROWS rows, one per thread, on its way to LDS.
template <int ROWS>
__device__ __forceinline__ float own_bias(const LogitsArgs& a, int64_t row0) {
    const int64_t row = row0 + threadIdx.x;
    return threadIdx.x < ROWS && a.bias && row < a.V ? a.bias[row] : 0.f;
}
// The logits of G hidden states from b0 on and a block's ROWS rows from row0 on, from LDS, where a hidden state is a row of ROWS + 4 floats.
// A wave writes whole rows of the block.  Memory takes lines of 64 bytes, and a part of one costs as much as many whole ones, so the 16-byte pieces
// that leave past the caches (which keep W and h) make up whole lines; what lies before the first line and after the last goes one by one
// through the cache, where the neighbour's part may still meet it.  2048 hidden states at 128257 x 128, float32, 4 bits / bf16: each wave its own
// 64 rows, in single logits, 436 / 427 us, so 221 / 317, and 208 where all rows start lines (V = 128256); 128257 x 4096 in 4 bits, bf16 logits, 662 -> 644.
// Products that are bound by the bf16 matrix rate lose up to 4 percent by it where V is odd, 1 percent at d = 4096.
template <int G, int ROWS, typename T>
__device__ __forceinline__ void give_out(const LogitsArgs& a, const float* buf, int64_t b0, int64_t row0) {
    constexpr int OW = ROWS + 4, E = 16 / sizeof(T), LINE = 4 * E, L = ROWS / E, P = 64 / L;      // lanes of a row, rows of a wave's pass
    static_assert(64 % L == 0 && G % (4 * P) == 0, "a wave takes whole rows");
    const int lane = threadIdx.x & 63, l = lane % L, n = (int)min((int64_t)ROWS, a.V - row0);
    for (int t = (threadIdx.x >> 6) * P + lane / L; t < G && b0 + t < a.B; t += 4 * P) {
        T* to = (T*)a.out + (b0 + t) * a.V + row0;
        const float* from = buf + t * OW;
        auto piece = [&](int e) {
            float v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = from[e + i];
            if constexpr (E == 4) __builtin_nontemporal_store(v4f{v[0], v[1], v[2], v[3]}, (v4f*)(to + e));
            else __builtin_nontemporal_store(v4u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}, (v4u*)(to + e));
        };
        if (a.lines) {
            if (l * E < n) piece(l * E);
            continue;
        }
        const int head = min(n, (int)(-(uintptr_t)to & 63) / (int)sizeof(T)), pieces = (n - head) / LINE * 4, singles = n - pieces * E;
        if (l < pieces) piece(head + l * E);
#pragma unroll
        for (int k = 0; k < (2 * LINE - 2 + L - 1) / L; ++k) {
            const int q = l + k * L, e = q < head ? q : q + pieces * E;
            if (q >= singles) continue;
            if constexpr (E == 4) to[e] = from[e];
            else to[e] = __builtin_bit_cast(uint16_t, (__bf16)from[e]);
        }
    }
}

// Codes that one block alone reads (ONCE: all hidden states in one group) go past the caches: 1 hidden state at a fresh head of 128256 x 4096
// 48.0 -> 42.6 us (the same head again 41.1 -> 40.5, with 30 of them 45.8 -> 48.5), 32 at 256000 x 4608 117 -> 105; where several blocks read them
// it costs as much (1024 at 128256 x 4096 in bf16 823 -> 878, 2048 1677 -> 1835).
template <bool ONCE>
__device__ __forceinline__ v4u load_codes(const uint8_t* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load((const v4u*)p);
    else return *(const v4u*)p;
}

// how the hidden states come: as they are, as 4-bit tiles, or to be rounded on the way to LDS
enum { H_BF16, H_TILES, H_ROUNDED_HERE };

// Four waves, RT tiles of 16 rows each, against NT groups of 16 hidden states; K goes by in stages of S tiles of 128.
//
// The sum over k may run in any order that both operands share.  A tile puts element 32 (l / 16) + 8 s + j at lane l, so a 4-bit tile goes to
// one 16x16x128 instruction as it is, and against bf16 it is widened (exactly) to four operands s = 0..3 of 16x16x32.
// Codes of W are read once, straight into registers, a stage ahead: a register is requested again as soon as its products are issued.  The
// stage of h lies in LDS, two buffers, and passes through registers on its way there, so that a barrier waits for no load.  bf16 h lies row by
// row with the 16-byte pieces of row t exchanged by t % 16 (a column of pieces then spreads over all banks); 4-bit h lies as its tiles, which few
// hidden states become here (a thread rounds a block: cheaper than a launch, while the block waits for W).
// Bound by the read of W up to 32 hidden states (64 in 4 bits): 1 at a fresh head of 128256 x 4096 42.6 us (6.6 TB/s), 32 at 256000 x 4608 with 33 MB of
// logits 105 us (6.3 TB/s); with more of them in bf16 by the matrix cores: 1024 at 128256 x 4096 824 us (1.3 PFLOP/s, the rate of the largest
// library products).
// Past the end of a row or of the batch the last piece or row is read again: the last stage puts zeros in the row's place, and those hidden
// states are not stored.
template <int H, int NT, int RT, int S, bool ONCE, typename T>
__global__ __launch_bounds__(256, 3) void product_kernel(LogitsArgs a) {
    constexpr bool MX4 = H != H_BF16, HERE = H == H_ROUNDED_HERE;
    constexpr int HP = NT * S * (MX4 ? 64 : 256);                 // 16-byte pieces of a stage of h
    constexpr int HT = (HP + 255) / 256;                          // of them per thread
    constexpr int ROWS = 64 * RT, OW = ROWS + 4;                  // floats per hidden state in the output buffer
    constexpr int GT = NT > 1 ? 2 : 1;                            // groups of hidden states that leave together
    constexpr int LDS = 2 * HP > GT * 4 * OW ? 2 * HP : GT * 4 * OW;
    __shared__ v4u lds[LDS];
    __shared__ v4f bias[ROWS / 4];
    __shared__ uint32_t hscale[HERE ? 2 * NT * 64 : 1];           // of h that is rounded here, a byte per step of the stage
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, col = lane & 15;
    // blocks of one die (every eighth) take the groups of hidden states of one block of rows after each other: W comes from that die's cache
    const int j = blockIdx.x >> 3, group = j % a.groups, block = (j / a.groups) * 8 + (blockIdx.x & 7);
    if (block >= a.blocks) return;
    const int chunks = a.chunks, quads = (chunks + 3) >> 2, stages = (chunks + S - 1) / S;
    const int64_t tile0 = (int64_t)block * (4 * RT) + wave * RT;
    const uint8_t* band = a.bands + (tile0 >> 2) * band_bytes(chunks);
    const uint8_t *wc = band + (tile0 & 3) * 1024 + lane * 16, *ws = band + (tile0 & 3) * 256 + lane * 4;
    const int64_t htile0 = (int64_t)group * NT;
    const uint32_t* hs = MX4 && !HERE ? a.hs + htile0 * quads * 64 + lane : nullptr;

    v4u w[S][RT], hr[HERE ? 4 * HT : HT];
    uint32_t sw[RT], sh[MX4 ? NT : 1], sw_next[RT], sh_next[MX4 ? NT : 1];
    auto load_w = [&](int c, v4u (&to)[RT]) {
        const int cc = min(c, chunks - 1);
#pragma unroll
        for (int r = 0; r < RT; ++r) to[r] = load_codes<ONCE>(wc + codes_at(cc) + r * 1024);
    };
    auto load_scales = [&](int c0) {                              // a stage lies within four tiles
        const int q = min(c0, chunks - 1) >> 2;
#pragma unroll
        for (int r = 0; r < RT; ++r) sw_next[r] = *(const uint32_t*)(ws + scales_at(q) + r * 256);
        if (MX4 && !HERE)
#pragma unroll
            for (int n = 0; n < NT; ++n) sh_next[n] = hs[((int64_t)n * quads + q) * 64];
    };
    auto load_h = [&](int c0) {
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int p = tid + i * 256;
            if (HP % 256 != 0 && p >= HP) continue;
            if constexpr (HERE) {                                 // block p / 16 % 4 of a step of hidden state p % 16: 64 bytes
                const int c = p / (NT * 64), n = p / 64 % NT, e = (c0 + c) * CHUNK + (p >> 4 & 3) * BLK;
                const int64_t b = min((int)(htile0 * 16) + n * 16 + (p & 15), a.B - 1);
#pragma unroll
                for (int k = 0; k < 4; ++k) hr[4 * i + k] = *(const v4u*)(a.h + b * a.d + min(e + 8 * k, a.d - 8));
            } else if constexpr (MX4) {
                const int c = p / (NT * 64), n = p / 64 % NT;
                hr[i] = ((const v4u*)a.hc)[((htile0 + n) * chunks + min(c0 + c, chunks - 1)) * 64 + (p & 63)];
            } else {
                const int c = p / (NT * 256), t = p / 16 % (NT * 16);
                const int64_t b = min((int)(htile0 * 16) + t, a.B - 1);
                hr[i] = *(const v4u*)(a.h + b * a.d + min((c0 + c) * CHUNK + (p & 15) * 8, a.d - 8));
            }
        }
    };
    auto store_h = [&](int buf, int c0, bool end) {
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int p = tid + i * 256;
            if (HP % 256 != 0 && p >= HP) continue;
            if constexpr (HERE) {
                const int c = p / (NT * 64), left = a.d - (c0 + c) * CHUNK - (p >> 4 & 3) * BLK;      // elements of the row from this block on
                uint32_t m = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (left <= 8 * k) hr[4 * i + k] = v4u{0, 0, 0, 0};
                    m = largest8(widen8(hr[4 * i + k]), m);
                }
                const uint32_t scale = scale_of(m);
                v4u codes;
#pragma unroll
                for (int k = 0; k < 4; ++k) codes[k] = codes8(widen8(hr[4 * i + k]), scale);
                lds[buf * HP + p] = codes;
                ((uint8_t*)hscale)[(buf * NT * 64 + p % (NT * 64)) * 4 + c] = (uint8_t)scale;
                continue;
            }
            // 0 times an infinity would be a NaN; whole steps behind the row are not multiplied
            if (!MX4 && end && (c0 + p / (NT * 256)) * CHUNK + (p & 15) * 8 >= a.d) hr[i] = v4u{0, 0, 0, 0};
            lds[buf * HP + (MX4 ? p : p ^ (p >> 4 & 15))] = hr[i];
        }
    };
    v4f acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = v4f{0.f, 0.f, 0.f, 0.f};
    auto products = [&](int buf, int c, const v4u (&x)[RT]) {
        const v4u* hb = lds + buf * HP + c * NT * (MX4 ? 64 : 256);
        if constexpr (MX4) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const v4u y = hb[n * 64 + lane];
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    acc[r][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widen(x[r]), widen(y), acc[r][n], 4, 4, 0, sw[r] >> (8 * c), 0, sh[n] >> (8 * c));
            }
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                v8bf wide[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) wide[r] = bf16_of_fp4(x[r][s], __uint_as_float((sw[r] >> (8 * c) & 255u) << 23));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const v8bf y = __builtin_bit_cast(v8bf, hb[(n * 16 + col) * 16 + ((4 * g + s) ^ col)]);
#pragma unroll
                    for (int r = 0; r < RT; ++r) acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[r], y, acc[r][n], 0, 0, 0);
                }
            }
        }
    };
    auto take_scales = [&](int c0) {
#pragma unroll
        for (int r = 0; r < RT; ++r) sw[r] = sw_next[r] >> (8 * (c0 & 3));
        if (MX4 && !HERE)
#pragma unroll
            for (int n = 0; n < NT; ++n) sh[n] = sh_next[n] >> (8 * (c0 & 3));
    };
    auto read_hscales = [&](int buf) {                            // after the barrier
        if (HERE)
#pragma unroll
            for (int n = 0; n < NT; ++n) sh[n] = hscale[(buf * NT + n) * 64 + lane];
    };

    load_h(0);
    load_scales(0);
#pragma unroll
    for (int c = 0; c < S; ++c) load_w(c, w[c]);
    for (int st = 0; st < stages - 1; ++st) {
        store_h(st & 1, st * S, false);
        take_scales(st * S);
        load_h((st + 1) * S);
        load_scales((st + 1) * S);
        lds_barrier();
        read_hscales(st & 1);
#pragma unroll
        for (int c = 0; c < S; ++c) {
            products(st & 1, c, w[c]);
            load_w((st + 1) * S + c, w[c]);
            __builtin_amdgcn_sched_barrier(0);                    // requests stay where they are written
        }
    }
    const int last = stages - 1;                                  // the last stage asks for nothing more
    store_h(last & 1, last * S, true);
    take_scales(last * S);
    lds_barrier();
    read_hscales(last & 1);
#pragma unroll
    for (int c = 0; c < S; ++c)
        if (last * S + c < chunks) products(last & 1, c, w[c]);

    // lane l holds rows 4 (l / 16) .. + 3 of hidden state l % 16 of every tile
    if (tid < ROWS) ((float*)bias)[tid] = own_bias<ROWS>(a, tile0 * 16 - wave * (RT * 16));
    __syncthreads();
    float* buf = (float*)lds;
#pragma unroll
    for (int n = 0; n < NT; n += GT) {
        const int64_t b0 = (htile0 + n) * 16;
        if (b0 >= a.B) break;                                     // of the whole block
        if (n > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int e = (wave * RT + r) * 16 + g * 4;
#pragma unroll
            for (int k = 0; k < GT; ++k) *(v4f*)(buf + (k * 16 + col) * OW + e) = acc[r][n + k] + bias[e >> 2];
        }
        __syncthreads();
        give_out<16 * GT, ROWS, T>(a, buf, b0, tile0 * 16 - wave * (RT * 16));
    }
}

// 256 rows against 128 hidden states in four bits, four waves of 64 rows, where there are enough of both: bound by the matrix cores.
// 32x32x64 instructions run at 1.7 times the rate of 16x16x128 (6.6 and 3.9 PFLOP/s measured on registers alone, random codes; what holds
// them at 6.6 is power: codes of zeros reach 8.9).  Lane l of theirs holds a block of row l % 32: two tiles side by side, read in
// pieces of 256 bytes, blocks l / 32 and then 2 + l / 32 of a step.
// The blocks that share a band ask for its codes at about the same time, so that each of them waits for memory, not for a cache.  Codes are
// therefore requested four steps ahead, each register again as soon as its products are issued; h comes two steps at a time, one such
// stage ahead, from global memory to LDS without registers, which are all taken: 128 sums, 64 of codes.  2048 at 128256 x 4096, bf16 logits: 602 to
// 617 us with the rounding of h, 9 of them (3.5 PFLOP/s; 640 for this kernel alone under a profiler, at a lower clock); matrix cores busy 46 % of the cycles.
// Before the logits left in whole lines, when a pass took 610 us, its parts, each taken away in turn, were: the
// writes of the logits 95 us, codes that come from memory 50, h from memory 20, all three 130; codes of zeros 85 (the clock, which random codes
// lower); products, LDS reads and barriers alone took 371.  Blocks twice as wide, groups of hidden states that stay in a cache and starts
// staggered so that writes meet other blocks' products gained nothing.
template <bool ONCE, typename T>
__global__ __launch_bounds__(256, 2) void many_kernel(LogitsArgs a) {
    constexpr int OW = 256 + 4;
    static_assert(32 * OW / 4 <= 2 * 1024 + 256, "logits take the place of h");
    __shared__ v4u lds[2 * 1024 + 256 + 64];                      // one array: with two the compiler waits for h on its way to LDS at every read
    v4f* bias = (v4f*)(lds + 2 * 1024 + 256);
    uint32_t* hscale = (uint32_t*)(lds + 2 * 1024);               // two buffers of 8 tiles
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // as in product_kernel, but the blocks of rows of a die are neighbours: they share lines of logits
    const int j = blockIdx.x >> 3, group = j % a.groups, block = (blockIdx.x & 7) * ((a.blocks + 7) >> 3) + j / a.groups;
    if (block >= a.blocks) return;
    const int chunks = a.chunks, quads = (chunks + 3) >> 2;
    const int at = (lane >> 4 & 1) * 64 + (lane >> 5) * 16 + (lane & 15);      // this lane's block in a run of tiles, in lanes
    auto step = [](int r) { return (r >> 1) * 128 + (r & 1) * 32; };           // and from there to register r: tiles 2 (r / 2), blocks 2 (r % 2)
    const uint8_t* band = a.bands + ((int64_t)block * 4 + wave) * band_bytes(chunks);
    const int64_t htile0 = (int64_t)group * 8;
    // addresses: a scalar for the wave and 32 bits for the lane
    const uint8_t* hc = a.hc + (htile0 + wave) * chunks * 1024;
    const uint8_t* hs = (const uint8_t*)a.hs + (htile0 + wave) * quads * 256;
    const uint32_t at16 = at * 16, at4 = at * 4, lane16 = lane * 16, lane4 = lane * 4;

    v4u w[4][4];
    uint32_t sw[4], sw_next[4];
    auto load_w = [&](int c, v4u (&to)[4]) {
        const uint8_t* p = band + codes_at(min(c, chunks - 1));
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] = load_codes<ONCE>(p + (at16 + step(r) * 16));
    };
    auto load_scales = [&](int q) {
        q = min(q, quads - 1);
        const uint8_t* p = band + scales_at(q);
#pragma unroll
        for (int r = 0; r < 4; ++r) sw_next[r] = *(const uint32_t*)(p + (at4 + step(r) * 4));
    };
    // h goes past the registers: wave w brings tiles w and w + 4, of two steps, or their scales of four.  (Buffer loads: global loads to LDS count
    // as loads that may touch either memory, and then every wait for a register waits for all of them.)
    typedef __attribute__((address_space(3))) void* lds_ptr;
    const auto h_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)hc, 0, 5 * chunks * 1024, 0x00027000);      // raw bytes, checked against the last tile's end
    const auto hs_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)hs, 0, 5 * quads * 256, 0x00027000);
    auto load_h = [&](int c0, int buf) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(h_rsrc, (lds_ptr)(lds + buf * 1024 + (i >> 1) * 512 + (i & 1) * 256 + wave * 64), 16, lane16,
                                                     ((i & 1) * 4 * chunks + min(c0 + (i >> 1), chunks - 1)) * 1024, 0, 0);
    };
    auto load_hscales = [&](int q) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(hs_rsrc, (lds_ptr)(hscale + (q & 1) * 512 + i * 256 + wave * 64), 4, lane4,
                                                     (i * 4 * quads + min(q, quads - 1)) * 256, 0, 0);
    };
    v16f acc[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][n][i] = 0.f;
    auto products = [&](auto step_c, int q, const v4u (&x)[4]) {
        constexpr int c = decltype(step_c)::value;
        const v4u* hb = lds + (c >> 1) * 1024 + (c & 1) * 512;
        const uint32_t* sb = hscale + (q & 1) * 512;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const v4u y = hb[at + step(n)];
            const uint32_t sy = sb[at + step(n)];
#pragma unroll
            for (int r = n & 1; r < 4; r += 2)
                acc[r >> 1][n >> 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(x[r]), widen(y), acc[r >> 1][n >> 1], 4, 4, c, sw[r], c, sy);
        }
    };
    // A stage of two steps: its h is in LDS, the next one's requested.  The eight loads of codes that follow h's are the youngest ones: waiting
    // for all but eight waits for h (and for the codes of this stage), not for codes of later ones.
    auto begin = [&](int q, int half, bool more) {
        // (A fence in place of the barrier's memory clobber would wait for all loads, because those of h write LDS.)
        if (more || half == 0) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // nothing has been asked for after h
        if (half == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) sw[r] = sw_next[r];
        }
        if (more || half == 0) load_h(4 * q + 2 * half + 2, half ^ 1);
        if (more && half == 0) {
            load_hscales(q + 1);
            load_scales(q + 1);
        }
        __builtin_amdgcn_sched_barrier(0);                        // requests stay where they are written
    };
    load_h(0, 0);
    load_hscales(0);
    load_scales(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < 4; ++c) load_w(c, w[c]);
    for (int q = 0; q < quads - 1; ++q) {
        begin(q, 0, true);
        products(std::integral_constant<int, 0>(), q, w[0]);
        load_w(4 * q + 4, w[0]);
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 1>(), q, w[1]);
        load_w(4 * q + 5, w[1]);
        __builtin_amdgcn_sched_barrier(0);
        begin(q, 1, true);
        products(std::integral_constant<int, 2>(), q, w[2]);
        load_w(4 * q + 6, w[2]);
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 3>(), q, w[3]);
        load_w(4 * q + 7, w[3]);
        __builtin_amdgcn_sched_barrier(0);
    }
    const int last = quads - 1, left = chunks - 4 * last;         // the last steps ask for nothing more
    begin(last, 0, false);
    products(std::integral_constant<int, 0>(), last, w[0]);
    if (left > 1) products(std::integral_constant<int, 1>(), last, w[1]);
    if (left > 2) {
        begin(last, 1, false);
        products(std::integral_constant<int, 2>(), last, w[2]);
        if (left > 3) products(std::integral_constant<int, 3>(), last, w[3]);
    }

    // lane l holds rows 8 i + 4 (l / 32) .. + 3 of hidden state l % 32 of a block of 32 x 32; h of a stage that was not needed may still be on its way
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    ((float*)bias)[tid] = own_bias<256>(a, (int64_t)block * 256);
    __syncthreads();
    float* buf = (float*)lds;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int64_t b0 = htile0 * 16 + n * 32;
        if (b0 >= a.B) break;                                     // of the whole block
        if (n > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = wave * 64 + r * 32 + i * 8 + (lane >> 5) * 4;
                *(v4f*)(buf + (lane & 31) * OW + e) = v4f{acc[r][n][4 * i], acc[r][n][4 * i + 1], acc[r][n][4 * i + 2], acc[r][n][4 * i + 3]} + bias[e >> 2];
            }
        __syncthreads();
        give_out<32, 256, T>(a, buf, b0, (int64_t)block * 256);
    }
}

// blocks of the grid for tiles of `rows` x `states`, or 0 where they are too many
static unsigned plan(LogitsArgs& a, int rows, int states) {
    a.blocks = (a.V + rows - 1) / rows;
    a.groups = (a.B + states - 1) / states;
    const int64_t n = (int64_t)(a.blocks + 7) / 8 * 8 * a.groups;
    if (n <= 0xffffff) return (unsigned)n;                       // a launch holds fewer than 2^32 threads
    csv_set_error("V=%d rows x B=%d hidden states are too many blocks", a.V, a.B);
    return 0;
}
template <int H, int NT, int RT, int S, bool ONCE>
static int launch_product(LogitsArgs a, int out_type, hipStream_t st) {
    const unsigned n = plan(a, 64 * RT, 16 * NT);
    if (!n) return CSV_ESHAPE;
    if (out_type == CSV_F32) product_kernel<H, NT, RT, S, ONCE, float><<<n, 256, 0, st>>>(a);
    else product_kernel<H, NT, RT, S, ONCE, uint16_t><<<n, 256, 0, st>>>(a);
    CSV_LAUNCH_CHECK("product_kernel");
    return CSV_OK;
}
template <bool ONCE>
static int launch_many(LogitsArgs a, int out_type, hipStream_t st) {
    const unsigned n = plan(a, 256, 128);
    if (!n) return CSV_ESHAPE;
    if (out_type == CSV_F32) many_kernel<ONCE, float><<<n, 256, 0, st>>>(a);
    else many_kernel<ONCE, uint16_t><<<n, 256, 0, st>>>(a);
    CSV_LAUNCH_CHECK("many_kernel");
    return CSV_OK;
}

// ------------------------------------------------------------------------------------------------ entry points
static int check_rows(int rows, int d, int type, int64_t ld, const void* x, const uint8_t* codes, const uint8_t* scales) {
    if (rows < 0 || d < 8 || (d & 7) != 0) { csv_set_error("need rows >= 0 and d a positive multiple of 8 (rows=%d, d=%d)", rows, d); return CSV_ESHAPE; }
    if (rows > 1 << 30 || d > 1 << 30) { csv_set_error("rows=%d or d=%d is above 2^30", rows, d); return CSV_ESHAPE; }
    if (type != CSV_F32 && type != CSV_BF16) { csv_set_error("bad element type %d", type); return CSV_EINVAL; }
    if (ld < d || (ld & 7) != 0) { csv_set_error("row stride %lld is below d=%d or no multiple of 8", (long long)ld, d); return CSV_ESHAPE; }
    if (rows == 0) return CSV_OK;
    if (!x || !codes || !scales) { csv_set_error("null rows, codes or scales"); return CSV_EINVAL; }
    if (((uintptr_t)x | (uintptr_t)codes) & 15) { csv_set_error("rows and codes have to be 16-byte aligned"); return CSV_EINVAL; }
    if ((uintptr_t)scales & 3) { csv_set_error("scales have to be 4-byte aligned"); return CSV_EINVAL; }
    return CSV_OK;
}

static dim3 rows_grid(int rows, int chunks) {
    const int64_t y = ((int64_t)rows + 3) / 4;
    return dim3((chunks + 3) / 4, (unsigned)(y < 32768 ? y : 32768));
}

extern "C" int csv_mx4_quantize(const void* d_x, int x_type, int64_t ld, int rows, int d, uint8_t* d_codes, uint8_t* d_scales, void* stream) {
    const int rc = check_rows(rows, d, x_type, ld, d_x, d_codes, d_scales);
    if (rc || rows == 0) return rc;
    const int chunks = chunks_of(d);
    const dim3 g = rows_grid(rows, chunks);
    if (x_type == CSV_F32) quantize_kernel<float, false><<<g, 256, 0, (hipStream_t)stream>>>((const float*)d_x, ld, rows, rows, d, chunks, d_codes, d_scales);
    else quantize_kernel<uint16_t, false><<<g, 256, 0, (hipStream_t)stream>>>((const uint16_t*)d_x, ld, rows, rows, d, chunks, d_codes, d_scales);
    CSV_LAUNCH_CHECK("quantize_kernel");
    return CSV_OK;
}

extern "C" int csv_mx4_dequantize(const uint8_t* d_codes, const uint8_t* d_scales, int rows, int d, void* d_x, int x_type, int64_t ld, void* stream) {
    const int rc = check_rows(rows, d, x_type, ld, d_x, d_codes, d_scales);
    if (rc || rows == 0) return rc;
    const int chunks = chunks_of(d);
    const dim3 g = rows_grid(rows, chunks);
    if (x_type == CSV_F32) dequantize_kernel<float><<<g, 256, 0, (hipStream_t)stream>>>(d_codes, d_scales, rows, d, chunks, (float*)d_x, ld);
    else dequantize_kernel<uint16_t><<<g, 256, 0, (hipStream_t)stream>>>(d_codes, d_scales, rows, d, chunks, (uint16_t*)d_x, ld);
    CSV_LAUNCH_CHECK("dequantize_kernel");
    return CSV_OK;
}

extern "C" int csv_mx4_head_create(const uint8_t* d_codes, const uint8_t* d_scales, const float* d_b, int V, int d, void* stream, csv_mx4_head** out) {
    if (!out) { csv_set_error("null out"); return CSV_EINVAL; }
    *out = nullptr;
    if (!d_codes || !d_scales) { csv_set_error("null codes or scales"); return CSV_EINVAL; }
    if (V < 1 || d < 8 || (d & 7) != 0) { csv_set_error("need V >= 1 and d a positive multiple of 8 (V=%d, d=%d)", V, d); return CSV_ESHAPE; }
    if (V > 0x7fffffff - HEAD_ROWS || d > CSV_MX4_MAX_D) { csv_set_error("V=%d or d=%d is too large", V, d); return CSV_ESHAPE; }
    if ((uintptr_t)d_codes & 15) { csv_set_error("codes have to be 16-byte aligned"); return CSV_EINVAL; }
    const int64_t bands = ((int64_t)V + HEAD_ROWS - 1) / HEAD_ROWS * (HEAD_ROWS / 64), pieces = bands * chunks_of(d) * 256;
    if (pieces > 0xffffff00LL) { csv_set_error("head of %d x %d: 2^37 padded elements or more", V, d); return CSV_ESHAPE; }
    csv_mx4_head* x = (csv_mx4_head*)calloc(1, sizeof(csv_mx4_head));
    if (!x) { csv_set_error("host allocation failed"); return CSV_ENOMEM; }
    x->V = V;
    x->d = d;
    x->chunks = chunks_of(d);
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipGetDevice(&x->device);
    if (e == hipSuccess) e = hipMalloc((void**)&x->bands, (size_t)(bands * band_bytes(x->chunks)));
    if (e == hipSuccess && d_b) e = hipMalloc((void**)&x->bias, (size_t)V * 4);
    if (e == hipSuccess && d_b) e = hipMemcpyAsync(x->bias, d_b, (size_t)V * 4, hipMemcpyDeviceToDevice, st);
    if (e == hipSuccess) {
        lay_out_kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(d_codes, d_scales, V, d, x->chunks, pieces, x->bands);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    if (e != hipSuccess) {
        csv_take_error();
        csv_set_error("head of %d x %d: %s", V, d, hipGetErrorString(e));
        csv_mx4_head_free(x);
        return e == hipErrorOutOfMemory ? CSV_ENOMEM : CSV_EHIP;
    }
    *out = x;
    return CSV_OK;
}

extern "C" int csv_mx4_head_dims(const csv_mx4_head* x, int* V, int* d) {
    if (!x) { csv_set_error("null head"); return CSV_EINVAL; }
    if (V) *V = x->V;
    if (d) *d = x->d;
    return CSV_OK;
}

extern "C" void csv_mx4_head_free(csv_mx4_head* x) {
    if (!x) return;
    void* ptrs[] = {x->bands, x->bias};
    for (void* p : ptrs)
        if (p) (void)hipFree(p);
    free(x);
}

static int check_logits(const csv_mx4_head* x, int B, int act) {
    if (!x) { csv_set_error("null head"); return CSV_EINVAL; }
    if (B < 0 || B > CSV_MX4_MAX_BATCH) { csv_set_error("B=%d outside 0..%d", B, CSV_MX4_MAX_BATCH); return CSV_ESHAPE; }
    if (act != CSV_ACT_BF16 && act != CSV_ACT_MX4) { csv_set_error("bad act=%d", act); return CSV_EINVAL; }
    return CSV_OK;
}
#define ROUNDED_HERE 16             // hidden states that the product rounds to 4 bits itself
// tiles of the 4-bit copy of h: a whole number of what a block of the product takes together
static inline int64_t tiles_of(int B) {
    const int64_t nt = B <= 32 ? 2 : B <= 64 ? 4 : 8;
    return ((int64_t)B + 16 * nt - 1) / (16 * nt) * nt;
}

extern "C" int csv_mx4_logits_scratch(const csv_mx4_head* x, int B, int act, size_t* bytes) {
    const int rc = check_logits(x, B, act);
    if (rc) return rc;
    if (!bytes) { csv_set_error("null bytes"); return CSV_EINVAL; }
    *bytes = act == CSV_ACT_BF16 || B <= ROUNDED_HERE ? 0 : (size_t)tiles_of(B) * ((size_t)x->chunks * 1024 + (size_t)((x->chunks + 3) / 4) * 256);
    return CSV_OK;
}

extern "C" int csv_mx4_logits(const csv_mx4_head* x, const uint16_t* d_h, int B, int act, void* d_logits, int out_type, void* d_scratch,
                              size_t scratch_bytes, void* stream) {
    size_t need = 0;
    const int rc = csv_mx4_logits_scratch(x, B, act, &need);
    if (rc) return rc;
    if (out_type != CSV_F32 && out_type != CSV_BF16) { csv_set_error("bad element type %d", out_type); return CSV_EINVAL; }
    if (B == 0) return CSV_OK;
    if (!d_h || !d_logits) { csv_set_error("null h or d_logits"); return CSV_EINVAL; }
    if ((uintptr_t)d_h & 15) { csv_set_error("h has to be 16-byte aligned"); return CSV_EINVAL; }
    if ((uintptr_t)d_logits & (out_type == CSV_F32 ? 3 : 1)) { csv_set_error("d_logits is not aligned to its type"); return CSV_EINVAL; }
    if (need && (!d_scratch || scratch_bytes < need)) { csv_set_error("scratch of %zu bytes, %zu are needed", d_scratch ? scratch_bytes : (size_t)0, need); return CSV_ESHAPE; }
    if (need && ((uintptr_t)d_scratch & 15)) { csv_set_error("scratch has to be 16-byte aligned"); return CSV_EINVAL; }
    int dev = -1;
    CSV_HIP(hipGetDevice(&dev));
    if (dev != x->device) { csv_set_error("the head lives on device %d, the current device is %d", x->device, dev); return CSV_EINVAL; }
    const hipStream_t st = (hipStream_t)stream;
    LogitsArgs a = {};
    a.bands = x->bands; a.bias = x->bias; a.V = x->V; a.d = x->d; a.chunks = x->chunks; a.B = B; a.h = d_h; a.out = d_logits;
    a.lines = ((uintptr_t)d_logits & 63) == 0 && x->V % (out_type == CSV_F32 ? 16 : 32) == 0;
    const int64_t tt = tiles_of(B);
    if (need) {
        uint8_t* hc = (uint8_t*)d_scratch;
        uint8_t* hs = hc + (size_t)tt * x->chunks * 1024;
        quantize_kernel<uint16_t, true><<<rows_grid((int)(tt * 16), x->chunks), 256, 0, st>>>(d_h, x->d, B, (int)(tt * 16), x->d, x->chunks, hc, hs);
        CSV_LAUNCH_CHECK("quantize_kernel");
        a.hc = hc;
        a.hs = (const uint32_t*)hs;
    }
    // Waves that take 64 rows each read h least often, waves of 32 rows make more blocks: below three blocks for two compute units
    // the units that have none, or two, cost more.  Microseconds, 32 / 64 rows a wave, from d = 4096: bf16, 14 hidden states, V = 80000
    // 32.5 / 36.3, 100000 42.1 / 39.3, 128256 48.1 / 44.9;  30 of them, 80000 38.3 / 41.0, 100000 48.9 / 43.2;  4 bits, 60, 80000 39.3 / 43.2,
    // 128256 55.9 / 52.7.  (16 rows: 32.9 and 54.5 for 14 at 80000 and 128256.)  At small heads, read again and again: 32000 x 1024, 1 hidden state
    // 4.8 / 6.3, 14 5.1 / 6.8;  64000 x 1024, 14, 7.6 / 7.9;  32000 x 4096, 14, 12.1 / 19.5;  50000 x 4096, 1, 20.9 / 23.7, 30, 25.4 / 23.1.
    const int64_t full = ((int64_t)x->V + 255) / 256;             // blocks of four waves of 64 rows
    const int64_t fill = 384;
    if (act == CSV_ACT_BF16) {
        if (B <= 16) return full >= fill ? launch_product<H_BF16, 1, 4, 2, true>(a, out_type, st) : launch_product<H_BF16, 1, 2, 4, true>(a, out_type, st);
        if (B <= 32) return full >= fill ? launch_product<H_BF16, 2, 4, 2, true>(a, out_type, st) : launch_product<H_BF16, 2, 2, 2, true>(a, out_type, st);
        // where groups of 64 make too few blocks, groups of 32 read W more often, from cache: 60 hidden states, 50000 x 4096, 36.2 against
        // 42.7, 128256 x 4096, 82.4 against 69.8.  Groups of 128 win nothing (817 against 832 for 1024): widening W is hidden behind the products
        if (full * ((B + 63) / 64) < fill) return launch_product<H_BF16, 2, 4, 2, false>(a, out_type, st);
        return B <= 64 ? launch_product<H_BF16, 4, 4, 1, true>(a, out_type, st) : launch_product<H_BF16, 4, 4, 1, false>(a, out_type, st);
    }
    if (B <= ROUNDED_HERE) return full >= fill ? launch_product<H_ROUNDED_HERE, 1, 4, 2, true>(a, out_type, st) : launch_product<H_ROUNDED_HERE, 1, 2, 4, true>(a, out_type, st);
    if (B <= 32) return launch_product<H_TILES, 2, 2, 4, true>(a, out_type, st);
    if (B <= 64) return full >= fill ? launch_product<H_TILES, 4, 4, 1, true>(a, out_type, st) : launch_product<H_TILES, 4, 2, 2, true>(a, out_type, st);
    // 100 hidden states: 24000 x 4096, 28.8 against 23.9 in groups of 64; 60000 x 2048, 22.7 against 26.8
    if (full * ((B + 127) / 128) < fill / 2) return launch_product<H_TILES, 4, 2, 2, false>(a, out_type, st);
    return B <= 128 ? launch_many<true>(a, out_type, st) : launch_many<false>(a, out_type, st);
}
