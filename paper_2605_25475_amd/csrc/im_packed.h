// The cache held in 4 bits, in pages: append, read back, attention with the memory readout, compaction, forks.
//
// A page holds IM_PAGE_SLOTS slots of one unit (batch element, KV head).  A row of 128 values is 128 codes of 4 bits (E2M1: sign and
// 0, 0.5, 1, 1.5, 2, 3, 4, 6; even dims in the low halves of the bytes) and one scale byte s per 32 dims: value = code 2^(s - 127).
// s = 255 marks a block that held an infinity or a NaN: all of it reads as NaN.  This is what the conversions and the scaled
// products of gfx950 take: a scale byte shifted to a float's exponent is their scale operand, 255 included.
//   bytes    0 .. 4095   K: row r at 64 r
//         4096 .. 8191   V: word w (dims 8 w .. 8 w + 7) of row r at 1024 (r / 16) + 16 (16 (r % 16 / 4) + w) + 4 (r % 4): a lane's
//                        share of 16 keys, 4 keys x 8 dims as the product P V takes them, is one 16-byte load
//         8192 .. 8447   K scales: block c of row r at 4 r + c
//         8448 .. 8703   V scales: block c of row r at 64 (r / 16) + 16 (r % 16 / 4) + 4 c + r % 4
#pragma once
#include "im_kernels.h"

#define PG_SLOTS 64
#define PG_BYTES 8704
#define PG_V 4096
#define PG_KS 8192
#define PG_VS 8448
#define IM_STATUS_OUT_OF_PAGES_BIT 16
#define IM_STATUS_BAD_FORK_BIT 32
#define IM_STATUS_BAD_PAGE_BIT 64
#define IM_STATUS_BAD_LISTS_BIT 128

typedef __bf16 im_bf2 __attribute__((ext_vector_type(2)));
typedef float im_f2 __attribute__((ext_vector_type(2)));
typedef float im_c16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ int pg_v_word(int r, int w) { return PG_V + (r >> 4) * 1024 + (((r & 15) >> 2) * 16 + w) * 16 + (r & 3) * 4; }
__device__ __forceinline__ int pg_v_scale(int r, int c) { return PG_VS + (r >> 4) * 64 + ((r & 15) >> 2) * 16 + c * 4 + (r & 3); }
__device__ __forceinline__ bool pg_is_page(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages; }
__device__ __forceinline__ float pg_scale(uint32_t s) { return __uint_as_float(s << 23); }

// 8 codes -> 8 bf16 values
__device__ __forceinline__ uint4 pg_expand(uint32_t w, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}

// the scale byte of a block from the largest |x| of its 32 values (bf16 patterns): the smallest s with |x| <= 6 * 2^(s - 127) (s >= 1):
// nothing is clipped.  With |x| = 1.m 2^e that is e - 2, and one more where 1.m > 1.5.
__device__ __forceinline__ uint32_t pg_scale_byte(uint32_t a) {
  return a >= 0x7f80u ? 255u : (uint32_t)max((int)(a >> 7) - 2 + ((a & 0x7f) > 0x40), 1);
}
__device__ __forceinline__ uint32_t pg_largest(uint4 x, uint32_t a) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) a = max(a, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  return a;
}
// 8 bf16 values -> a code word; to the nearest code, ties to the even one
__device__ __forceinline__ uint32_t pg_codes(uint4 x, uint32_t s) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const float f = pg_scale(s);
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = bf_lo(w[i]); v[2 * i + 1] = bf_hi(w[i]); }
  if (s == 253u) {   // 4 * 2^126 is no bf16 value: what is nearest to it goes to 3 * 2^126
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(v[i], -0x1.8p127f), 0x1.8p127f);
  }
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], f, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], f, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], f, 3);
  return s == 255u ? 0u : q;
}

// word k of 34 (16 of K, 16 of V, K's scales, V's scales) of a row, from one page's row to another's
__device__ __forceinline__ void pg_copy_word(const char* src, int rs, char* dst, int rd, int k) {
  if (k < 16) *(uint32_t*)(dst + rd * 64 + 4 * k) = *(const uint32_t*)(src + rs * 64 + 4 * k);
  else if (k < 32) *(uint32_t*)(dst + pg_v_word(rd, k - 16)) = *(const uint32_t*)(src + pg_v_word(rs, k - 16));
  else if (k == 32) *(uint32_t*)(dst + PG_KS + 4 * rd) = *(const uint32_t*)(src + PG_KS + 4 * rs);
  else if (k == 33) {
#pragma unroll
    for (int c = 0; c < 4; ++c) dst[pg_v_scale(rd, c)] = src[pg_v_scale(rs, c)];
  }
}

// ------------------------------------------------------------------------------------------
// pages: who needs one, and which are free
// ------------------------------------------------------------------------------------------
// exclusive sum over the 1024 threads of a workgroup; total in every thread.  Every thread calls it.
__device__ __forceinline__ int pg_scan(int v, int* s_wave, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int inc = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  __syncthreads();   // (s_wave of the call before has been read)
  if (lane == 63) s_wave[w] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int t = s_wave[i];
    before += i < w ? t : 0;
    total += t;
  }
  return before + inc - v;
}

// The lowest `want` free pages (refs = 0), ascending, to ids; returns how many there are of them.  One workgroup.
#define PG_LOOK 16   // pages a thread looks at together
__device__ __forceinline__ int pg_find_free(const int32_t* __restrict__ refs, int n_pages, int want, int32_t* ids, int* s_wave) {
  int found = 0;
  for (long long p0 = 0; p0 < n_pages && found < want; p0 += 1024 * PG_LOOK) {
    const long long p = p0 + PG_LOOK * threadIdx.x;
    uint32_t f = 0;
    int total, users[PG_LOOK];   // (all loads are on their way together)
    if (p + PG_LOOK <= n_pages) {
      __builtin_memcpy(users, refs + p, sizeof(users));
    } else {
#pragma unroll
      for (int i = 0; i < PG_LOOK; ++i) users[i] = p + i < n_pages ? refs[p + i] : 1;
    }
#pragma unroll
    for (int i = 0; i < PG_LOOK; ++i) f |= users[i] == 0 ? 1u << i : 0u;
    int at = found + pg_scan(__popc(f), s_wave, total);
    for (; f && at < want; f &= f - 1) ids[at++] = (int)p + __ffs(f) - 1;
    found += total;
  }
  return min(found, want);
}

// The scratch of the two launches of an append or a compaction (ints in the workspace): per unit [units] each, per page of a unit [units * T]
struct PgScratch {
  int32_t *base, *cow, *end;   // append: old length or -1; page to copy from or -1; compaction: 1 if the unit is compacted
  int32_t *rank, *free_ids, *old;
};

// Append, first launch: one workgroup.  Item (unit, i) is the i-th page that the unit's new tokens touch.  A page is needed where the
// table has none, or where others hold it too (then the entries in front of the new ones are copied by the second launch).  Pages go
// to the items in order, the lowest free one first; a unit whose pages are not all there is left as it is.  A chain of memory round trips:
// 2.2 us for 32 units, 4.5 where a page is taken; 8 units x 4096 tokens with every page to take 3.1; 10 with 32768 used pages in front of the free ones.
__global__ __launch_bounds__(1024) void k_packed_plan_append(int32_t* __restrict__ table, int32_t* __restrict__ refs, int n_pages,
                                                             int32_t* __restrict__ len, int32_t* __restrict__ n_projected, int units,
                                                             int T, int C, int n_new, PgScratch ws, int32_t* __restrict__ status) {
  __shared__ int s_wave[16];
  const uint32_t P = min((n_new - 1) / PG_SLOTS + 2, T), tid = threadIdx.x, items = (uint32_t)units * P;
  int want = 0;
  for (uint32_t i0 = 0; i0 < items; i0 += 1024) {
    const uint32_t i = i0 + tid, u = i / P, k = i - u * P;
    int need = 0;
    if (i < items) {
      const int n = len[u], p = n / PG_SLOTS + (int)k;
      if (n >= 0 && n <= C - n_new && p <= (n + n_new - 1) / PG_SLOTS) {
        const int page = table[(size_t)u * T + p];
        need = !pg_is_page(page, n_pages) || refs[page] > 1;
      }
    }
    int total;
    const int before = pg_scan(need, s_wave, total);
    if (i < items) {
      ws.rank[i] = need ? want + before : -1;
      if (k == P - 1) ws.end[u] = want + before + need;
    }
    want += total;
  }
  __syncthreads();
  const int found = want ? pg_find_free(refs, n_pages, want, ws.free_ids, s_wave) : 0;
  __syncthreads();
  for (int u = tid; u < units; u += 1024) {
    const int n = len[u], end = ws.end[u], begin = u ? ws.end[u - 1] : 0;
    const bool room = n >= 0 && n <= C - n_new, pages = end == begin || end <= found;
    if (!room) atomicOr(status, IM_STATUS_APPEND_OVERFLOW_BIT);
    else if (!pages) atomicOr(status, IM_STATUS_OUT_OF_PAGES_BIT);
    ws.base[u] = room && pages ? n : -1;
    ws.cow[u] = -1;
    if (room && pages) len[u] = n_projected[u] = n + n_new;
  }
  if (want == 0) return;
  __syncthreads();
  for (uint32_t i = tid; i < items; i += 1024) {
    const uint32_t u = i / P, k = i - u * P;
    const int n = ws.base[u], r = ws.rank[i];
    if (n < 0 || r < 0) continue;
    const int id = ws.free_ids[r];
    int32_t* entry = &table[(size_t)u * T + n / PG_SLOTS + k];
    const int old = *entry;
    *entry = id;
    refs[id] = 1;
    if (pg_is_page(old, n_pages)) {
      atomicSub(&refs[old], 1);
      if (k == 0 && n % PG_SLOTS) ws.cow[u] = old;
    }
  }
}

// Append, second launch, up to 4 new rows: grid (2, units), 256 threads.  Workgroup 0 rounds and stores the rows (16 lanes a row, a
// quad of lanes a block), workgroup 1 makes the indexer keys: neither waits for the other's loads.  4.2 us for 32 units, the chain of the key's
// fp64 projection and norm.
__device__ __forceinline__ void pg_copy_page_head(char* pages, const int32_t* tab, const PgScratch& ws, int unit, int base) {
  if (ws.cow[unit] < 0) return;   // the entries of a shared page in front of the new ones
  const char* src = pages + (size_t)ws.cow[unit] * PG_BYTES;
  char* dst = pages + (size_t)tab[base / PG_SLOTS] * PG_BYTES;
  for (int i = threadIdx.x; i < base % PG_SLOTS * 34; i += 256) pg_copy_word(src, i / 34, dst, i / 34, i % 34);
}
__global__ __launch_bounds__(256) void k_packed_append_few(char* __restrict__ pages, const int32_t* __restrict__ table, int T,
                                                           bf16_t* __restrict__ Kidx, int32_t* __restrict__ pos,
                                                           const bf16_t* __restrict__ k_new, const bf16_t* __restrict__ v_new,
                                                           const int32_t* __restrict__ pos_new, int n_new, int H_kv, int C,
                                                           const bf16_t* __restrict__ Uk, const bf16_t* __restrict__ norm_w,
                                                           float rms_eps, PgScratch ws) {
  __shared__ ProjectSmem sm;
  const int unit = blockIdx.y, tid = threadIdx.x, l16 = tid & 15, row = tid >> 4, base = ws.base[unit];
  const bf16_t *K = k_new + (size_t)unit * n_new * IM_D, *V = v_new + (size_t)unit * n_new * IM_D;
  if (base < 0) return;
  if (blockIdx.x == 1) {   // (from the rows as they were given: the unit's rows and keys from its first new one on)
    project_keys_few(K, Kidx + ((size_t)unit * C + base) * IM_DI, Uk, norm_w, 0, rms_eps, 0, 0, n_new, sm);
    return;
  }
  const int32_t* tab = table + (size_t)unit * T;
  pg_copy_page_head(pages, tab, ws, unit, base);
  if (row >= n_new) return;   // (rows are quads of lanes)
  const uint4 k = *(const uint4*)(K + row * IM_D + 8 * l16), v = *(const uint4*)(V + row * IM_D + 8 * l16);
  auto quad_max = [](uint32_t a) {
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)a, 0xB1, 0xF, 0xF, false));      // quad_perm 1 0 3 2
    return max(a, (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)a, 0x4E, 0xF, 0xF, false));   // quad_perm 2 3 0 1
  };
  const uint32_t ks = pg_scale_byte(quad_max(pg_largest(k, 0))), vs = pg_scale_byte(quad_max(pg_largest(v, 0)));
  const int slot = base + row, r = slot % PG_SLOTS;
  char* page = pages + (size_t)tab[slot / PG_SLOTS] * PG_BYTES;
  *(uint32_t*)(page + r * 64 + 4 * l16) = pg_codes(k, ks);
  *(uint32_t*)(page + pg_v_word(r, l16)) = pg_codes(v, vs);
  if (l16 % 4 == 0) {
    page[PG_KS + 4 * r + l16 / 4] = (char)ks;
    page[pg_v_scale(r, l16 / 4)] = (char)vs;
  }
  if (l16 == 0) pos[(size_t)unit * C + slot] = pos_new[(size_t)(unit / H_kv) * n_new + row];
}

// The same for more rows: grid (tiles of 64 new rows, units), 4 waves of 16 rows.  Lane (l16, kq) has dims 32 kq .. 32 kq + 31 of row l16, a
// block of its own, as the key projection takes them: a row is read once, and rounded while the projection's products run.  8 units x 4096 rows:
// 19 us, one generation of workgroups, each a chain of loads, products (7 us at the fp64 matrix cores' peak; without them 14 us), norm, rounding
// and stores; 32 units x 4096 rows 59 us, 3.2 TB/s (at 3 waves per SIMD instead of 4: 61, though at 4 the compiler spills 5 registers of a
// lane, 24 bytes).  (Rounding and projection as workgroups of their
// own: twice the time.)
__global__ __launch_bounds__(256, 4) void k_packed_append(char* __restrict__ pages, const int32_t* __restrict__ table, int T,
                                                       bf16_t* __restrict__ Kidx, int32_t* __restrict__ pos,
                                                       const bf16_t* __restrict__ k_new, const bf16_t* __restrict__ v_new,
                                                       const int32_t* __restrict__ pos_new, int n_new, int H_kv, int C,
                                                       const bf16_t* __restrict__ Uk, const bf16_t* __restrict__ norm_w, float rms_eps,
                                                       PgScratch ws) {
  __shared__ ProjectSmem sm;
  const int unit = blockIdx.y, lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
  const int row0 = blockIdx.x * 64 + 16 * (threadIdx.x >> 6), row = row0 + l16;
  const size_t at = ((size_t)unit * n_new + min(row, n_new - 1)) * IM_D + 32 * kq;
  uint4 k[4], v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k[i] = load_stream16(k_new + at + 8 * i);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = load_stream16(v_new + at + 8 * i);
  const int base = ws.base[unit];
  if (base < 0) return;
  const int32_t* tab = table + (size_t)unit * T;
  if (blockIdx.x == 0) pg_copy_page_head(pages, tab, ws, unit, base);
  if (row0 >= n_new) return;   // (wave-uniform; no workgroup barrier below)
  const int slot = base + min(row, n_new - 1), r = slot % PG_SLOTS;
  char* page = pages + (size_t)tab[slot / PG_SLOTS] * PG_BYTES;
  project_keys_rows(k, Kidx + ((size_t)unit * C + base + row0) * IM_DI, Uk, norm_w, rms_eps, min(16, n_new - row0), sm);
  uint32_t ka = 0, va = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) { ka = pg_largest(k[i], ka); va = pg_largest(v[i], va); }
  const uint32_t ks = pg_scale_byte(ka), vs = pg_scale_byte(va);
  if (row < n_new) {
    *(uint4*)(page + r * 64 + 16 * kq) = make_uint4(pg_codes(k[0], ks), pg_codes(k[1], ks), pg_codes(k[2], ks), pg_codes(k[3], ks));
#pragma unroll
    for (int i = 0; i < 4; ++i) *(uint32_t*)(page + pg_v_word(r, 4 * kq + i)) = pg_codes(v[i], vs);
    page[PG_KS + 4 * r + kq] = (char)ks;
    page[pg_v_scale(r, kq)] = (char)vs;
    if (kq == 0) pos[(size_t)unit * C + slot] = pos_new[(size_t)(unit / H_kv) * n_new + row];
  }
}

// Read back: grid (gx, units), 16 lanes per row.  idx NULL: every entry of the unit.  Bound by memory, four fifths of it writes: 32 units x
// 14336 rows 69 us, 4.36 TB/s (a copy reaches 5.1).
__global__ __launch_bounds__(256) void k_packed_unpack(const char* __restrict__ pages, int n_pages, const int32_t* __restrict__ table, int T,
                                                       const int32_t* __restrict__ len, int C, const int32_t* __restrict__ idx,
                                                       const int32_t* __restrict__ n_idx, bf16_t* __restrict__ K,
                                                       bf16_t* __restrict__ V, int32_t* __restrict__ status) {
  const int unit = blockIdx.y, l16 = threadIdx.x & 15, live = min(len[unit], C);
  const int n = idx ? min(n_idx[unit], C) : live;
  const int32_t* tab = table + (size_t)unit * T;
  // (4 rows at a time: 71.5 us instead of 68.4 for 4 x 8 units x 14336 rows)
  for (int i = blockIdx.x * 16 + (threadIdx.x >> 4); i < n; i += gridDim.x * 16) {
    const int slot = idx ? idx[(size_t)unit * C + i] : i;
    if (slot < 0 || slot >= live) continue;
    const int page_id = tab[slot / PG_SLOTS], r = slot % PG_SLOTS;
    if (!pg_is_page(page_id, n_pages)) {
      if (l16 == 0) atomicOr(status, IM_STATUS_BAD_PAGE_BIT);
      continue;
    }
    const char* page = pages + (size_t)page_id * PG_BYTES;
    const uint32_t kw = *(const uint32_t*)(page + r * 64 + 4 * l16), vw = *(const uint32_t*)(page + pg_v_word(r, l16));
    const float ks = pg_scale((uint8_t)page[PG_KS + 4 * r + l16 / 4]), vs = pg_scale((uint8_t)page[pg_v_scale(r, l16 / 4)]);
    const size_t at = ((size_t)unit * C + slot) * IM_D + 8 * l16;
    *(uint4*)(K + at) = pg_expand(kw, ks);
    *(uint4*)(V + at) = pg_expand(vw, vs);
  }
}

// ------------------------------------------------------------------------------------------
// attention of few rows per unit (n_q queries x G heads)
// ------------------------------------------------------------------------------------------
struct PgAttn {
  const char* pages;
  const int32_t *table, *len, *pos;
  const bf16_t* q;
  const int32_t* q_pos;   // NULL: every query sees every entry
  float* part;            // records [batch][query][head][split]: maximum (of log2), denominator, 128 numerators
  int32_t* status;
  int n_pages, T, C, H, H_kv, G, n_q, max_live, n_splits;
  float scale;
};
#define PG_REC (IM_D + 2)
#define PG_NO_MAX (-3e38f)   // the maximum of a row that has seen nothing: below it no entry is told from none

// m c2, the reference of a row's weights exp2(s c2 - m c2): its rounding is a factor of all of them, and goes out in the quotient.  Where the
// logits are so far from 0 that the factor leaves the weights' range (2^22: it is 2^(1/4) at most), pg_far is true, and s - m, which is exact for
// those that count, takes the place of s
__device__ __forceinline__ float pg_reference(float m, float c2) { return fmaxf(m * c2, PG_NO_MAX); }
__device__ __forceinline__ bool pg_far(float m, float mc) { return m > PG_NO_MAX && fabsf(mc) > 0x1p22f; }

// p[block][tile][r] of 32 keys (row 16 block + l16, key 16 tile + 4 kq + r) times V; the probabilities go in as two bf16 parts (16 bits:
// 2^-17 of each, where one part would cost as much as the output's own rounding), o accumulates in fp32
template <int NB>
__device__ __forceinline__ void pg_pv(const float (&p)[NB][2][4], const uint4 (&vf)[2][4], im_c4 (&o)[NB][8]) {
  im_bf8 ph[NB], pl[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{p[x][t][2 * h], p[x][t][2 * h + 1]}), im_bf2));
        hi[2 * t + h] = w;
        lo[2 * t + h] = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{p[x][t][2 * h] - bf_lo(w), p[x][t][2 * h + 1] - bf_hi(w)}), im_bf2));
      }
    ph[x] = __builtin_bit_cast(im_bf8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    pl[x] = __builtin_bit_cast(im_bf8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const im_bf8 v = att_column(vf, e);
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      o[x][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl[x], v, o[x][e], 0, 0, 0);
      o[x][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ph[x], v, o[x][e], 0, 0, 0);
    }
  }
}

// grid (splits, units, tiles of 16 NB rows), 4 waves; a wave takes one page in four of its split: the logits of 64 keys as 4 tiles of 16 x 16
// for each block of 16 rows (keys x rows; row r is query r / G, head r % G), the softmax against a running maximum, P V.  A page is expanded once
// for the NB blocks, in registers: its layout is that of the products' operands.  The waves' sums meet in LDS.
//   One query of 4 heads over 8 units x 131072 entries: 31 us, 4.6 TB/s, bound by memory (a copy reaches 5.1).  16 units x 7 heads x 2048: 9.4 us.
// With 32 rows (NB 2) the products and the softmax are in front: 20 rows over 64 units x 16384 entries 56 us.  Two blocks' logits, sums and queries and the next
// page's bytes are more than 256 registers: the compiler spills 22 of a lane with the mask (92 bytes), 6 without (28).
template <bool MASK, int NB>
__global__ __launch_bounds__(256, 2) void k_packed_attn_few(PgAttn a) {
  __shared__ float s_ml[4][16 * NB][2];
  __shared__ uint32_t s_nan[4][16 * NB];
  __shared__ __attribute__((aligned(16))) float s_acc[4][16 * NB][IM_D];
  const int unit = blockIdx.y, split = blockIdx.x, b = unit / a.H_kv, h = unit % a.H_kv;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, kq = lane >> 4, l16 = lane & 15;
  const int n_true = a.len[unit], n = min(n_true, a.max_live), r0 = blockIdx.z * 16 * NB, R = min(16 * NB, a.n_q * a.G - r0);
  if (n_true > a.max_live && split == 0 && tid == 0) atomicOr(a.status, IM_STATUS_LIVE_EXCEEDED_BIT);
  const int n_pages = (n + PG_SLOTS - 1) / PG_SLOTS, per = (n_pages + a.n_splits - 1) / a.n_splits;
  const int p_end = min(n_pages, (split + 1) * per);
  uint4 qf[NB][4];
  int q_pos[NB], q_lo = 0x7fffffff;   // what every row sees is not above q_lo
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const int row = r0 + min(16 * x + l16, R - 1), query = row / a.G;
    const size_t q_row = ((size_t)b * a.n_q + query) * a.H + h * a.G + row % a.G;
#pragma unroll
    for (int c = 0; c < 4; ++c) qf[x][c] = *(const uint4*)(a.q + q_row * IM_D + 32 * kq + 8 * c);
    q_pos[x] = MASK ? a.q_pos[(size_t)b * a.n_q + query] : 0;
    q_lo = min(q_lo, q_pos[x]);
  }
  const int32_t* tab = a.table + (size_t)unit * a.T;
  const float c2 = a.scale * 1.44269504088896340736f;   // exp(scale x) = exp2(c2 x)
  float m[NB], l[NB];
  uint32_t nan_blocks[NB];
  im_c4 o[NB][8];
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    m[x] = PG_NO_MAX;
    l[x] = 0.f;
    nan_blocks[x] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[x][e] = im_c4{0.f, 0.f, 0.f, 0.f};
  }
  // the next page's bytes are on their way while a page is worked on
  uint4 kw[4], vw[4], kw_next[4], vw_next[4];
  uint32_t ks[4], vs[4], ks_next[4], vs_next[4];
  int ps = 0, ps_next = 0;   // position of the page's entry `lane`
  if (MASK) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) q_lo = min(q_lo, __shfl_xor(q_lo, d, 64));
  }
  auto fetch = [&](int p) {   // false: a table entry that names no page: nothing is there
    const int id = tab[p];
    if (!pg_is_page(id, a.n_pages)) {
      if (lane == 0) atomicOr(a.status, IM_STATUS_BAD_PAGE_BIT);
      return false;
    }
    const char* page = a.pages + (size_t)id * PG_BYTES;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      kw_next[t] = load_stream16(page + 1024 * t + 64 * l16 + 16 * kq);
      ks_next[t] = (uint8_t)page[PG_KS + 64 * t + 4 * l16 + kq];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      vw_next[t] = load_stream16(page + PG_V + 1024 * t + 16 * lane);
      vs_next[t] = *(const uint32_t*)(page + PG_VS + 64 * t + 16 * kq + 4 * (l16 >> 2));
    }
    if (MASK) ps_next = a.pos[(size_t)unit * a.C + min(p * PG_SLOTS + lane, n - 1)];
    return true;
  };
  int p = split * per + w;
  bool there = p < p_end && fetch(p);
  for (; p < p_end; p += 4) {
    const bool now = there;
#pragma unroll
    for (int t = 0; t < 4; ++t) { kw[t] = kw_next[t]; vw[t] = vw_next[t]; ks[t] = ks_next[t]; vs[t] = vs_next[t]; }
    ps = ps_next;
    there = p + 4 < p_end && fetch(p + 4);
    if (!now) continue;
    const int nk = min(PG_SLOTS, n - p * PG_SLOTS);
    float s[NB][4][4], top[NB];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float f = pg_scale(ks[t]);
      const uint4 kf[4] = {pg_expand(kw[t].x, f), pg_expand(kw[t].y, f), pg_expand(kw[t].z, f), pg_expand(kw[t].w, f)};
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const im_c4 acc = att_logits(kf, qf[x]);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[x][t][r] = acc[r];
      }
    }
    if (nk < PG_SLOTS || (MASK && __any(ps > q_lo))) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = 16 * t + 4 * kq + r;
          const int at = MASK ? __shfl(ps, key, 64) : 0;   // (every lane takes part)
#pragma unroll
          for (int x = 0; x < NB; ++x) s[x][t][r] = key < nk && (!MASK || at <= q_pos[x]) ? s[x][t][r] : -INFINITY;
        }
    }
    bool larger = false;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      top[x] = s[x][0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) top[x] = fmaxf(top[x], s[x][t][r]);
      top[x] = rows_max_f(top[x]);
      larger |= (top[x] - m[x]) * c2 > 8.f;
    }
    if (__any(larger)) {   // (P may grow to 2^8 before the maximum follows)
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const float m_new = fmaxf(m[x], top[x]), f = __builtin_amdgcn_exp2f((m[x] - m_new) * c2);
        m[x] = m_new;
        l[x] *= f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {   // the rows of o lie across the lane groups, their factors in lanes 0 .. 15
          const float fr = __shfl(f, 4 * kq + r, 64);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[x][e][r] *= fr;
        }
      }
    }
    float mc[NB];
    bool far = false;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      mc[x] = pg_reference(m[x], c2);
      far |= pg_far(m[x], mc[x]);
    }
    if (__any(far)) {
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        mc[x] = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[x][t][r] -= m[x];
      }
    }
#pragma unroll
    for (int x = 0; x < NB; ++x) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[x][t][r] = __builtin_amdgcn_exp2f(fmaf(s[x][t][r], c2, -mc[x]));
          l[x] += s[x][t][r];
        }
    }
    // entries behind the last one hold anything: their values are taken as 0; a block of NaN among the others would reach rows that do
    // not see it (0 * NaN): it is taken as 0, too, and remembered for the rows that do
    bool has_255 = false;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t y = ~vs[t];
      has_255 |= ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
    }
    if (nk < PG_SLOTS || __any(has_255)) {
      bool odd = false;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t wv[4] = {vw[t].x, vw[t].y, vw[t].z, vw[t].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool live = 16 * t + 4 * kq + i < nk, nan = ((vs[t] >> (8 * i)) & 255u) == 255u;
          odd |= live && nan;
          if (!live || nan) { wv[i] = 0u; vs[t] &= ~(255u << (8 * i)); }
        }
        vw[t] = make_uint4(wv[0], wv[1], wv[2], wv[3]);
      }
      if (__any(odd)) {
        const char* page = a.pages + (size_t)tab[p] * PG_BYTES;
        for (int key = 0; key < nk; ++key) {
          uint32_t blocks = 0;
          for (int c = 0; c < 4; ++c) blocks |= (uint8_t)page[pg_v_scale(key, c)] == 255u ? 1u << c : 0u;
#pragma unroll
          for (int x = 0; x < NB; ++x)
            if (blocks && (!MASK || a.pos[(size_t)unit * a.C + p * PG_SLOTS + key] <= q_pos[x])) nan_blocks[x] |= blocks;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint4 vf[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint4 x = vw[2 * t + u];
        const uint32_t wv[4] = {x.x, x.y, x.z, x.w}, b4 = vs[2 * t + u];
        const uint32_t sc[4] = {b4 << 23, (b4 << 15) & 0x7f800000u, (b4 << 7) & 0x7f800000u, (b4 >> 1) & 0x7f800000u};
#pragma unroll
        for (int i = 0; i < 4; ++i) vf[u][i] = pg_expand(wv[i], __uint_as_float(sc[i]));
      }
      float pr[NB][2][4];
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) pr[x][u][r] = s[x][2 * t + u][r];
      pg_pv<NB>(pr, vf, o);
    }
  }
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    l[x] = rows_sum_f(l[x]);
    if (kq == 0) { s_ml[w][16 * x + l16][0] = pg_reference(m[x], c2); s_ml[w][16 * x + l16][1] = l[x]; s_nan[w][16 * x + l16] = nan_blocks[x]; }
    if (R > 16 * x) att_store(o[x], &s_acc[w][16 * x][0], l16, kq, min(R - 16 * x, 16));
  }
  __syncthreads();
  for (int i = tid; i < R * IM_D; i += 256) {
    const int r = i >> 7, d = i & 127;
    const float mm = fmaxf(fmaxf(s_ml[0][r][0], s_ml[1][r][0]), fmaxf(s_ml[2][r][0], s_ml[3][r][0]));
    float ov = 0.f, lv = 0.f;
    uint32_t nb = 0;
#pragma unroll
    for (int ww = 0; ww < 4; ++ww) {
      const float f = __builtin_amdgcn_exp2f(s_ml[ww][r][0] - mm);
      ov = fmaf(f, s_acc[ww][r][d], ov);
      lv = fmaf(f, s_ml[ww][r][1], lv);
      nb |= s_nan[ww][r];
    }
    if ((nb >> (d >> 5)) & 1u) ov = NAN;
    const size_t rec_row = ((size_t)b * a.n_q + (r0 + r) / a.G) * a.H + h * a.G + (r0 + r) % a.G;
    float* rec = a.part + (rec_row * a.n_splits + split) * PG_REC;
    rec[2 + d] = ov;
    if (d == 0) { rec[0] = mm; rec[1] = lv; }
  }
}

// The splits of a row joined, and the gated memory readout added: grid (ceil(n_q G / RW), units), 512 threads, RW rows of a unit per
// workgroup.  Thread (x, g) has column x of the memory in rows 32 g .. 32 g + 31, row x of Wtheta in dims 32 g .. 32 g + 31, and of the
// splits every fourth: four short chains that meet in LDS, instead of one of 128 steps.  A chain of memory round trips and barriers: 4.7 us for
// 32 rows of 2 to 64 splits.
template <int RW>
__global__ __launch_bounds__(512) void k_packed_combine(const float* __restrict__ part, int n_splits, const bf16_t* __restrict__ q,
                                                        const bf16_t* __restrict__ Wtheta, const bf16_t* __restrict__ wg, float cg,
                                                        const float* __restrict__ M, const float* __restrict__ bvec, int H, int H_kv,
                                                        int G, int n_q, float mem_eps, bf16_t* __restrict__ out,
                                                        float* __restrict__ readout_dbg) {
  __shared__ float s_q[RW][IM_D], s_phi[RW][IM_DM], s_sum[4][RW][IM_D], s_o[4][RW][IM_D], s_ml[4][RW][2], s_red[RW][2][2];
  const int unit = blockIdx.y, b = unit / H_kv, h = unit % H_kv, tid = threadIdx.x, x = tid & 127, g = tid >> 7;
  const int r0 = blockIdx.x * RW, R = n_q * G;
  auto row_of = [&](int i) {   // row i of the workgroup, in [batch][query][head]; rows behind the last repeat it
    const int r = min(r0 + i, R - 1);
    return ((size_t)b * n_q + r / G) * H + h * G + r % G;
  };
  float mcol[32];
  const float* Mu = M + ((size_t)unit * IM_DM + 32 * g) * IM_D + x;
#pragma unroll
  for (int c = 0; c < 32; ++c) mcol[c] = Mu[c * IM_D];
  uint4 wrow[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) wrow[i] = *(const uint4*)(Wtheta + x * IM_D + 32 * g + 8 * i);
  const float bv = bvec[(size_t)unit * IM_DM + x], wgv = bf2f(wg[x]);
#pragma unroll
  for (int i = 0; i < RW; ++i)
    if (i % 4 == g) s_q[i][x] = bf2f(q[row_of(i) * IM_D + x]);
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    const float* rec = part + row_of(i) * n_splits * PG_REC;
    float m = PG_NO_MAX, l = 0.f, o = 0.f;
    for (int c0 = g; c0 < n_splits; c0 += 32) {   // 8 splits at a time
      float cm[8], cl[8], co[8], top = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float* p = rec + (size_t)min(c0 + 4 * j, n_splits - 1) * PG_REC;
        cm[j] = p[0]; cl[j] = p[1]; co[j] = p[2 + x];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c0 + 4 * j < n_splits) top = fmaxf(top, cm[j]);
      const float f = __builtin_amdgcn_exp2f(m - top);
      l *= f; o *= f; m = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (c0 + 4 * j < n_splits) {
          const float e = __builtin_amdgcn_exp2f(cm[j] - m);
          l = fmaf(e, cl[j], l);
          o = fmaf(e, co[j], o);
        }
      }
    }
    s_o[g][i][x] = o;
    if (x == 0) { s_ml[g][i][0] = m; s_ml[g][i][1] = l; }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    float ph = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u[4] = {wrow[j].x, wrow[j].y, wrow[j].z, wrow[j].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ph = fmaf(bf_lo(u[e]), s_q[i][32 * g + 8 * j + 2 * e], ph);
        ph = fmaf(bf_hi(u[e]), s_q[i][32 * g + 8 * j + 2 * e + 1], ph);
      }
    }
    s_sum[g][i][x] = ph;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RW; ++i)
    if (i % 4 == g) {
      const float ph = (s_sum[0][i][x] + s_sum[1][i][x]) + (s_sum[2][i][x] + s_sum[3][i][x]);
      s_phi[i][x] = ph;
      const float den = wave_sum_f(ph * ph * bv), gz = wave_sum_f(wgv * s_q[i][x]);
      if ((tid & 63) == 0) { s_red[i][x >> 6][0] = den; s_red[i][x >> 6][1] = gz; }
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    float mr = 0.f;
#pragma unroll
    for (int c = 0; c < 32; ++c) mr = fmaf(s_phi[i][32 * g + c], mcol[c], mr);
    s_sum[g][i][x] = mr;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RW; ++i)
    if (i % 4 == g && r0 + i < R) {
      const float m = fmaxf(fmaxf(s_ml[0][i][0], s_ml[1][i][0]), fmaxf(s_ml[2][i][0], s_ml[3][i][0]));
      float o = 0.f, l = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(s_ml[k][i][0] - m);
        o = fmaf(f, s_o[k][i][x], o);
        l = fmaf(f, s_ml[k][i][1], l);
      }
      const float den = s_red[i][0][0] + s_red[i][1][0] + mem_eps, gz = s_red[i][0][1] + s_red[i][1][1] + cg;
      const float mr = (s_sum[0][i][x] + s_sum[1][i][x]) + (s_sum[2][i][x] + s_sum[3][i][x]);
      const float res = 1.f / (1.f + __expf(-gz)) * (mr / den);
      const size_t at = row_of(i) * IM_D + x;
      out[at] = f2bf_rne((l == 0.f ? 0.f : o / l) + res);   // (no entry seen: 0)
      if (readout_dbg) readout_dbg[at] = res;
    }
}

// ------------------------------------------------------------------------------------------
// attention of many rows
// ------------------------------------------------------------------------------------------
#define PG_ROWS 128        // rows of a workgroup: 32 per wave
#define PG_SEG 512         // pages whose masks are looked at together

struct PgReadout {
  const bf16_t *Wtheta, *wg;
  const float *M, *b;
  float cg, mem_eps;
  bf16_t* out;
  float* readout;   // the whole output is written to out, and the readout here if not NULL; with several splits the readout alone, by the first
};

__device__ __forceinline__ im_c16 pg_zero16() {
  im_c16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
__device__ __forceinline__ float halves_max_f(float v) {
  typedef unsigned int u2 __attribute__((ext_vector_type(2)));
  const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// 8 floats as bf16 operands: nearest, and nearest of what is left
__device__ __forceinline__ void pg_split8(const float (&x)[8], im_bf8& hi, im_bf8& lo) {
  uint32_t a[4], r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{x[2 * i], x[2 * i + 1]}), im_bf2));
    r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{x[2 * i] - bf_lo(a[i]), x[2 * i + 1] - bf_hi(a[i])}), im_bf2));
  }
  hi = __builtin_bit_cast(im_bf8, make_uint4(a[0], a[1], a[2], a[3]));
  lo = __builtin_bit_cast(im_bf8, make_uint4(r[0], r[1], r[2], r[3]));
}

typedef _Float16 im_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 im_h2 __attribute__((ext_vector_type(2)));

// A page expanded in LDS.  16-byte piece g of K's row r (16 pieces) is at 16 (16 r + (g ^ r % 16)), of V's dim d (8 pieces of 8 keys) at
// 16 (8 d + (g ^ (d / 2 ^ d / 16) % 8)): the 16 rows that a read takes at a time (0-3, 12-15, 20-23, 24-27 of 32) fall on all 64
// banks, and the addresses of a thread's pieces are one value XOR constants.
#define PG_TILE 32768
#define PG_TILE_V 16384   // V behind K
struct PgTile {   // what goes with a tile
  __attribute__((aligned(16))) int pos[PG_SLOTS];
  int odd[4];   // whether the wave's 16 keys hold a block of NaN
};

// 4 keys x 8 dims of V (a word of codes and a scale byte per key) -> 8 pieces of 4 keys, fp16 values in units of 2^(e - 127); unit = 2^(127 - e).
// Exact for scales of e - 23 .. e + 13 (the smallest value is 0.5 x 2^-23, the largest 6 x 2^13 < 65504); a scale byte of 0 gives 0.
#define PG_BELOW 23
#define PG_ABOVE 13
#define PG_BAND (PG_BELOW + PG_ABOVE + 1)
__device__ __forceinline__ void pg_v_pieces(const uint4& vw, uint32_t vs, float unit, uint2 (&piece)[8]) {
  const uint32_t w[4] = {vw.x, vw.y, vw.z, vw.w}, sc[4] = {vs << 23, (vs << 15) & 0x7f800000u, (vs << 7) & 0x7f800000u, (vs >> 1) & 0x7f800000u};
  uint32_t x[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = __uint_as_float(sc[i]) * unit;
    x[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], f, 0));
    x[i][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], f, 1));
    x[i][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], f, 2));
    x[i][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[i], f, 3));
  }
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    const uint32_t sel = (d & 1) ? 0x07060302u : 0x05040100u;
    piece[d] = make_uint2(__builtin_amdgcn_perm(x[1][d >> 1], x[0][d >> 1], sel), __builtin_amdgcn_perm(x[3][d >> 1], x[2][d >> 1], sel));
  }
}

// grid (row tiles x splits x units), 4 waves; wave w has rows 32 w .. 32 w + 31 of the tile (row r is query r / G, head r % G) as the
// columns of every product, so that a lane's 16 logits of a block of 32 keys, its running maximum and its sums belong to one row:
//   S^T = K Q^T, O^T = V^T P^T; products of 32 x 32 x 16, register i of lane (l32, half) is row 8 (i / 4) + 4 half + i % 4, column l32.
// P^T's registers are its operand as they are; V^T's keys are laid out in LDS in that order (16 t + 8 half + 4 g + j for key
// 16 t + 8 g + 4 half + j).  A page of 64 keys is expanded in LDS by the whole workgroup, between the products S^T of the page before it, and the
// bytes of the page behind it are on their way.  (8 waves of 256 rows, half of them expanding K and half V: 470 us where this takes 473.)
//   K goes in as bf16 (exact).  2^7 P goes in as fp16, half a step of 2^-11 off each (the sums of P stay fp32), or 2^-32 where P is below 2^-21:
// 2^17 entries of a flat tail together are 2^-15 off (without the 2^7: 2^-8).  V goes in as fp16 multiples of a power of two per 32 dims, which the
// first segment's scales give: exact while all scales are among the 37 around it.  A segment with others is gone over once for every 37 powers of
// two that its scales span (up to 7 times), in units of their own, and what was summed up in the units before waits in private memory, as sums of
// the values themselves: fp32 holds these from 2^-126 up to entries of 2^96, whichever of them a row sees.  (V as bf16 and P as two bf16 parts:
// 48 products a page instead of 32.  The products of a page from 0, added to sums of the values in the loop: 560 us instead of 488, registers.)
//   4096 queries x 4 heads over 8 units x 8192 entries, causal: 474 us, 888 TFLOP/s of what the mask leaves (1389 in a large library product).
// The vector instructions of the softmax and the expansion (half of the cycles) and the products (36 %) share two waves per SIMD, that 256
// registers and the tiles allow; 56 us are the lists, the readout and the output.
__global__ __launch_bounds__(256, 2) void k_packed_attn_many(PgAttn a, PgReadout ro, int units) {
  __shared__ __attribute__((aligned(16))) char s_tile[2 * PG_TILE];
  __shared__ PgTile s_extra[2];
  __shared__ int s_list[PG_SEG];   // pages to look at; bit 31: some row does not see all of it
  __shared__ int s_n, s_lim[4][2], s_scale[4][4][2];
  // the units of a row tile side by side: with 8 of them, or a multiple, a unit's workgroups share an XCD's L2; the last rows, which see the
  // most of a prompt, first
  const int unit = blockIdx.x % units, split = blockIdx.x / units % a.n_splits, tile = gridDim.x / (units * a.n_splits) - 1 - blockIdx.x / (units * a.n_splits);
  const int b = unit / a.H_kv, h = unit % a.H_kv;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
  const int n_true = a.len[unit], n = min(n_true, a.max_live), R = a.n_q * a.G;
  if (n_true > a.max_live && split == 0 && tile == 0 && tid == 0) atomicOr(a.status, IM_STATUS_LIVE_EXCEEDED_BIT);
  const int n_pages = (n + PG_SLOTS - 1) / PG_SLOTS, per = (n_pages + a.n_splits - 1) / a.n_splits;
  const int p_begin = split * per, p_end = min(n_pages, p_begin + per);
  const int my_row = tile * PG_ROWS + 32 * w + l32, row = min(my_row, R - 1), query = row / a.G;
  const size_t q_row = ((size_t)b * a.n_q + query) * a.H + h * a.G + row % a.G;
  im_bf8 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) qf[s] = __builtin_bit_cast(im_bf8, *(const uint4*)(a.q + q_row * IM_D + 16 * s + 8 * half));
  const int q_pos = a.q_pos ? a.q_pos[(size_t)b * a.n_q + query] : 0x7fffffff;
  // the range of the tile's query positions
  {
    int lo = q_pos, hi = q_pos;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { lo = min(lo, __shfl_xor(lo, d, 64)); hi = max(hi, __shfl_xor(hi, d, 64)); }
    if (lane == 0) { s_lim[w][0] = lo; s_lim[w][1] = hi; }
  }
  __syncthreads();
  int q_lo = s_lim[0][0], q_hi = s_lim[0][1];
#pragma unroll
  for (int i = 1; i < 4; ++i) { q_lo = min(q_lo, s_lim[i][0]); q_hi = max(q_hi, s_lim[i][1]); }
  const int32_t *tab = a.table + (size_t)unit * a.T, *pos = a.pos + (size_t)unit * a.C;
  const float c2 = a.scale * 1.44269504088896340736f;   // exp(scale x) = exp2(c2 x)
  float m = PG_NO_MAX, l = 0.f;
  uint32_t nan_blocks = 0;
  int e_of[4] = {0, 0, 0, 0};   // o[d] counts 2^7 P V in 2^(e_of[d] - 127); 0: no values yet
  im_c16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] = pg_zero16();

  // a thread's share of a page: 32 codes of K (row tid / 4, block tid % 4), and of V (keys 16 w + 4 kq .. + 3, dims 8 l16 ..)
  const int l16 = lane & 15, kq = lane >> 4;
  // (LDS addresses as offsets in s_tile; they change tiles by an XOR with the tile's size)
  uint32_t k_put = 256 * (tid >> 2) + 16 * ((4 * (tid & 3)) ^ ((tid >> 2) & 15));
  uint32_t v_put = PG_TILE_V + 1024 * l16 + 16 * ((2 * w + (kq & 1)) ^ (4 * (l16 & 1)) ^ (l16 >> 1)) + 8 * (kq >> 1);
  uint32_t k_get = 256 * l32 + 16 * (half ^ (l32 & 15)), v_get = PG_TILE_V + 128 * l32 + 16 * (half ^ ((l32 >> 1) & 7) ^ (l32 >> 4));
  uint4 kw, vw;
  uint32_t ks, vs;
  int ps = 0;
  auto fetch = [&](int p) {   // (p is uniform: the page's address is in scalar registers, the thread's offset in one that stays)
    const char* page = a.pages + (size_t)tab[p] * PG_BYTES;
    kw = *(const uint4*)(page + 16 * tid);
    vw = *(const uint4*)(page + PG_V + 16 * tid);
    ks = (uint8_t)page[PG_KS + tid];
    vs = *(const uint32_t*)(page + PG_VS + 64 * w + 16 * kq + 4 * (l16 >> 2));
    if (a.q_pos) ps = pos[min(p * PG_SLOTS + lane, n - 1)];
  };

  // the listed pages; my_e: the units of this thread's share of V (2^(my_e - 127)); bands: times that the segment is gone over, this is the band-th,
  // with the PG_BAND scales up to my_top
  auto segment = [&](int count, int my_e, int my_top, int band, int bands) {
    const float unit = pg_scale(254 - max(my_e, 1));   // 2^(127 - my_e)
    // Entries behind the last one hold anything: their values are taken as 0, as a block of NaN is, which the rows that see it get below,
    // and what belongs to another band.  Whether there is NaN among these.
    auto settle = [&](int p) {
      const int nk = n - p * PG_SLOTS;
      const uint32_t y = ~vs;
      const bool has_255 = ((y - 0x01010101u) & ~y & 0x80808080u) != 0;   // some byte of vs is 255
      bool odd = false;
      if (nk < PG_SLOTS || bands > 1 || __any(has_255)) {
        uint32_t sc = vs;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t byte = (vs >> (8 * i)) & 255u;
          const bool live = 16 * w + 4 * kq + i < nk, nan = byte == 255u;
          odd |= live && nan;
          if (!live || nan || (bands > 1 && (uint32_t)(my_top - (int)byte) >= PG_BAND)) sc &= ~(255u << (8 * i));
        }
        vs = sc;
      }
      return __any(odd);
    };
    auto expand = [&](bool odd, PgTile& t) {
      const float f = pg_scale(ks);
      const uint32_t kv[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) *(uint4*)((char*)s_tile + (k_put ^ (16 * i))) = pg_expand(kv[i], f);
      uint2 piece[8];
      pg_v_pieces(vw, vs, unit, piece);
#pragma unroll
      for (int e = 0; e < 8; ++e) *(uint2*)((char*)s_tile + (v_put ^ (16 * (e >> 1))) + 128 * e) = piece[e];
      k_put ^= PG_TILE;
      v_put ^= PG_TILE;
      t.pos[lane] = ps;   // (every wave the same)
      t.odd[w] = odd;
    };
    auto entry_at = [&](int i) { return __builtin_amdgcn_readfirstlane(s_list[min(i, count - 1)]); };   // (the last one again where there are no more)
    auto page_at = [&](int i) { return entry_at(i) & 0x7fffffff; };
    fetch(page_at(0));
    expand(settle(page_at(0)), s_extra[0]);
    fetch(page_at(1));
    __syncthreads();
    for (int i = 0; i < count; ++i) {
      const PgTile& t = s_extra[i & 1];
      const int entry = entry_at(i), p = entry & 0x7fffffff, nk = n - p * PG_SLOTS;
      const bool odd_next = settle(page_at(i + 1));
      im_c16 sc[2];
      sc[0] = pg_zero16();
      sc[1] = pg_zero16();
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const char* at = (const char*)s_tile + (k_get ^ (32 * s));
#pragma unroll
        for (int u = 0; u < 2; ++u)
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(im_bf8, *(const uint4*)(at + 8192 * u)), qf[s], sc[u], 0, 0, 0);
      }
      k_get ^= PG_TILE;
      expand(odd_next, s_extra[(i & 1) ^ 1]);
      fetch(page_at(i + 2));
      if (entry < 0) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int key = 32 * u + 8 * g + 4 * half;
            int4 at = make_int4(0, 0, 0, 0);
            if (a.q_pos) at = *(const int4*)&t.pos[key];
            sc[u][4 * g + 0] = key + 0 < nk && at.x <= q_pos ? sc[u][4 * g + 0] : -INFINITY;
            sc[u][4 * g + 1] = key + 1 < nk && at.y <= q_pos ? sc[u][4 * g + 1] : -INFINITY;
            sc[u][4 * g + 2] = key + 2 < nk && at.z <= q_pos ? sc[u][4 * g + 2] : -INFINITY;
            sc[u][4 * g + 3] = key + 3 < nk && at.w <= q_pos ? sc[u][4 * g + 3] : -INFINITY;
          }
      }
      float top = sc[0][0];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[u][r]);
      top = halves_max_f(top);
      // (P may grow to 2^8 before the maximum follows: most pages bring some row a new one, few a much larger one)
      if (__any((top - m) * c2 > 8.f)) {
        const float m_new = fmaxf(m, top), f = __builtin_amdgcn_exp2f((m - m_new) * c2);
        m = m_new;
        l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= f;
      }
      float mc = pg_reference(m, c2) - 7.f;
      if (__any(pg_far(m, mc))) {
        mc = -7.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[u][r] -= m;
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 4; ++u) {   // 16 keys
        uint32_t x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = 8 * (u & 1) + 2 * r;
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[u >> 1][at], c2, -mc)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[u >> 1][at + 1], c2, -mc));
          const im_h2 pk = __builtin_convertvector((im_f2{p0, p1}), im_h2);
          sum[r & 1] = __builtin_amdgcn_fdot2(pk, im_h2{(_Float16)1.f, (_Float16)1.f}, sum[r & 1], false);   // (the sums of P as it goes in, in fp32)
          x[r] = __builtin_bit_cast(uint32_t, pk);
        }
        const im_h8 pf = __builtin_bit_cast(im_h8, make_uint4(x[0], x[1], x[2], x[3]));
#pragma unroll
        for (int d = 0; d < 4; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(im_h8, *(const uint4*)((const char*)s_tile + 4096 * d + (v_get ^ (32 * (u ^ d))))), pf, o[d], 0, 0, 0);
      }
      v_get ^= PG_TILE;
      l += band == 0 ? sum[0] + sum[1] : 0.f;
      if (t.odd[0] | t.odd[1] | t.odd[2] | t.odd[3]) {   // blocks of NaN: for the rows that see them
        const char* page = a.pages + (size_t)tab[p] * PG_BYTES;
        for (int key = 0; key < min(nk, PG_SLOTS); ++key) {
          uint32_t blocks = 0;
          for (int c = 0; c < 4; ++c) blocks |= (uint8_t)page[pg_v_scale(key, c)] == 255u ? 1u << c : 0u;
          if (blocks && (!a.q_pos || t.pos[key] <= q_pos)) nan_blocks |= blocks;
        }
      }
      __syncthreads();
    }
    k_put ^= PG_TILE;   // (writing was a tile ahead of reading)
    v_put ^= PG_TILE;
  };

  // what o holds goes to the sums that wait (2^7 of P are 2^(134 - 127)), which follow the maximum.  (In memory by the compiler's own word: registers
  // are what the loop over the pages lacks.)
  float by_memory[65];
  typedef __attribute__((address_space(5))) volatile float by_float;
  by_float* by = (by_float*)by_memory;
  bool waits = false;
  auto put_by = [&]() {
    if (!waits) {
#pragma unroll
      for (int i = 0; i < 64; ++i) by[i] = 0.f;
      by[64] = m;
    }
    const float f = __builtin_amdgcn_exp2f((by[64] - m) * c2);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        by[16 * d + r] = fmaf(by[16 * d + r], f, ldexpf(o[d][r], e_of[d] - 134));
        o[d][r] = 0.f;
      }
      e_of[d] = 0;
    }
    by[64] = m;
    waits = true;
  };

  for (int seg = p_begin; seg < p_end; seg += PG_SEG) {
    const int n_seg = min(PG_SEG, p_end - seg);
    // which pages the tile's rows see, which of them whole, and the largest and smallest scale (above 1, which is as good as 0) of their
    // values per block: lane (key / 4, block) looks at 4 keys; 4 pages of a wave at a time
    int s_hi = 0, s_lo = 255;
    __syncthreads();
    // wave w takes pages 8 w .. 8 w + 7 of every 32, all of their bytes together; lane j of a wave knows the number of its j-th page
    const int my_page = seg + min(32 * (lane >> 3) + 8 * w + (lane & 7), n_seg - 1);
    const int ids_a = tab[my_page], ids_b = n_seg > 256 ? tab[min(my_page + 256, seg + n_seg - 1)] : 0;
    for (int i0 = 8 * w, k = 0; i0 < n_seg; i0 += 32, k += 8) {
      int id[8], at[8];
      uint32_t sv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        id[j] = k < 64 ? __builtin_amdgcn_readlane(ids_a, (k + j) & 63) : __builtin_amdgcn_readlane(ids_b, (k + j) & 63);
        if (!pg_is_page(id[j], a.n_pages)) id[j] = -1;   // (a table entry that names no page: nothing is there)
        const char* page = a.pages + (size_t)max(id[j], 0) * PG_BYTES;
        sv[j] = *(const uint32_t*)(page + PG_VS + 4 * lane);
        at[j] = a.q_pos ? pos[min((seg + min(i0 + j, n_seg - 1)) * PG_SLOTS + lane, n - 1)] : 0;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = i0 + j, first = (seg + i) * PG_SLOTS;
        if (i >= n_seg) break;
        int entry = seg + i;
        if (first + PG_SLOTS > n) entry |= 1 << 31;
        if (a.q_pos) {
          const bool live = first + lane < n;
          if (!__any(live && at[j] <= q_hi)) entry = -1;
          else if (__any(live && at[j] > q_lo)) entry |= 1 << 31;
        }
        if (id[j] < 0) {
          if (lane == 0) atomicOr(a.status, IM_STATUS_BAD_PAGE_BIT);
          entry = -1;
        }
        if (lane == 0) s_list[i] = entry;
        if (entry == -1) continue;
#pragma unroll
        for (int b4 = 0; b4 < 4; ++b4) {
          const int byte = (sv[j] >> (8 * b4)) & 255u;
          const bool counts = byte != 255 && byte > 1 && first + 4 * (lane >> 2) + b4 < n;
          s_hi = counts ? max(s_hi, byte) : s_hi;
          s_lo = counts ? min(s_lo, byte) : s_lo;
        }
      }
    }
#pragma unroll
    for (int d = 4; d < 64; d <<= 1) { s_hi = max(s_hi, __shfl_xor(s_hi, d, 64)); s_lo = min(s_lo, __shfl_xor(s_lo, d, 64)); }
    if (lane < 4) { s_scale[w][lane][0] = s_hi; s_scale[w][lane][1] = s_lo; }
    __syncthreads();
    if (w == 0) {   // those that nobody sees leave the list
      int count = 0;
      for (int i0 = 0; i0 < n_seg; i0 += 64) {
        const int entry = i0 + lane < n_seg ? s_list[i0 + lane] : -1;
        const unsigned long long there = __ballot(entry != -1);
        if (entry != -1) s_list[count + __popcll(there & ((1ull << lane) - 1ull))] = entry;
        count += __popcll(there);
      }
      if (lane == 0) s_n = count;
    }
    __syncthreads();
    const int count = s_n;
    if (count == 0) continue;
    int bands = 1;
    for (int band = 0; band < bands; ++band) {
      int top[4], low[4];   // the scales of the band; top -PG_BAND: there are none, all are taken as 0
      bool fit = true;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        int hi = 0, lo = 255;
#pragma unroll
        for (int i = 0; i < 4; ++i) { hi = max(hi, s_scale[i][d][0]); lo = min(lo, s_scale[i][d][1]); }
        hi = __builtin_amdgcn_readfirstlane(hi);
        lo = __builtin_amdgcn_readfirstlane(lo);
        bands = hi > 0 ? max(bands, (hi - lo) / PG_BAND + 1) : bands;
        top[d] = hi - PG_BAND * band;
        if (hi == 0 || top[d] < lo) top[d] = -PG_BAND;
        low[d] = max(lo, top[d] - PG_BAND + 1);
        fit = fit && (top[d] < 0 || e_of[d] == 0 || (top[d] <= e_of[d] + PG_ABOVE && low[d] >= e_of[d] - PG_BELOW));
      }
      if (!fit) put_by();
#pragma unroll
      for (int d = 0; d < 4; ++d)   // (the first units leave room for larger scales to come, where they can)
        if (top[d] > 0 && e_of[d] == 0) e_of[d] = max(top[d] - (top[d] - low[d] < PG_BAND - 6 ? PG_ABOVE - 6 : PG_ABOVE), 1);
      const int my_d = l16 >> 2, my_e = my_d & 2 ? (my_d & 1 ? e_of[3] : e_of[2]) : (my_d & 1 ? e_of[1] : e_of[0]);
      const int my_top = my_d & 2 ? (my_d & 1 ? top[3] : top[2]) : (my_d & 1 ? top[1] : top[0]);
      segment(count, my_e > 0 ? my_e : 127, my_top, band, bands);   // (no units: what is there is 0, or as good as 0)
    }
  }
  if (waits) {
    put_by();
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = by[16 * d + r];
      e_of[d] = 134;
    }
  }
  l = halves_sum_f(l) * 0x1p-7f;
  const float to_o = a.n_splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;   // (no entry seen: 0)
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = ldexpf(o[d][r] * to_o, e_of[d] - 134);

  if (a.n_splits > 1) {   // the row's record; the splits are joined by k_packed_join
    if (my_row < R) {
      float* rec = a.part + (q_row * a.n_splits + split) * PG_REC;
      if (half == 0) { rec[0] = pg_reference(m, c2); rec[1] = l; }
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          rec[2 + 32 * d + 8 * (r >> 2) + 4 * half + (r & 3)] = (nan_blocks >> d) & 1u ? NAN : o[d][r];
    }
    if (split > 0) return;
  }

  // the memory readout of the wave's rows: phi^T = Wtheta Q^T, then M^T phi^T with phi and M as two bf16 parts each (2^-16).  Wtheta, then M's parts go
  // through LDS, once for the four waves (each reading them from the cache by itself: 20 us more of 16384 rows x 8 units): row r's 16-byte
  // piece g at 16 (16 r + (g ^ r % 16)), M by dims with its rows in the order of phi's registers.
  const float* Mu = ro.M + (size_t)unit * IM_DM * IM_D;
  auto piece_at = [&](int r, int g) { return s_tile + 256 * r + 16 * (g ^ (r & 15)); };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = tid + 256 * i;
    *(uint4*)piece_at(at >> 4, at & 15) = *(const uint4*)(ro.Wtheta + 8 * at);
  }
  float den = 0.f, gz = 0.f;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const uint4 x = __builtin_bit_cast(uint4, qf[s]), y = *(const uint4*)(ro.wg + 16 * s + 8 * half);
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) gz = fmaf(bf_lo(xw[e]), bf_lo(yw[e]), fmaf(bf_hi(xw[e]), bf_hi(yw[e]), gz));
  }
  __syncthreads();
  im_bf8 ph[8], pl[8];   // operand of 16 values of phi each
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) {
    im_c16 phi = pg_zero16();
#pragma unroll
    for (int s = 0; s < 8; ++s)
      phi = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(im_bf8, *(const uint4*)piece_at(32 * cb + l32, 2 * s + half)), qf[s], phi, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) den = fmaf(phi[r] * phi[r], ro.b[(size_t)unit * IM_DM + 32 * cb + 8 * (r >> 2) + 4 * half + (r & 3)], den);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) x[r] = phi[8 * t + r];
      pg_split8(x, ph[2 * cb + t], pl[2 * cb + t]);
    }
  }
  den = halves_sum_f(den) + ro.mem_eps;
  const float gate = 1.f / (1.f + __expf(-(halves_sum_f(gz) + ro.cg))) / den;
  __syncthreads();
  // rows 4 c .. 4 c + 3 of M, of one dim: half of piece 2 (c / 4) + c % 2, its first half for c % 4 < 2
#pragma unroll 4
  for (int i = 0; i < 16; ++i) {
    const int dim = tid & 127, c = 2 * i + (tid >> 7);
    float x[4];
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = Mu[(4 * c + r) * IM_D + dim];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      hi[r] = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{x[2 * r], x[2 * r + 1]}), im_bf2));
      lo[r] = __builtin_bit_cast(uint32_t, __builtin_convertvector((im_f2{x[2 * r] - bf_lo(hi[r]), x[2 * r + 1] - bf_hi(hi[r])}), im_bf2));
    }
    char* at = piece_at(dim, 2 * (c >> 2) + (c & 1)) + 8 * ((c >> 1) & 1);
    *(uint2*)at = make_uint2(hi[0], hi[1]);
    *(uint2*)(at + PG_TILE) = make_uint2(lo[0], lo[1]);
  }
  __syncthreads();
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    im_c16 mem = pg_zero16();
#pragma unroll
    for (int t = 0; t < 8; ++t) {   // 16 of the memory's rows
      const char* at = piece_at(32 * d + l32, 2 * t + half);
      const im_bf8 mh = __builtin_bit_cast(im_bf8, *(const uint4*)at), ml = __builtin_bit_cast(im_bf8, *(const uint4*)(at + PG_TILE));
      mem = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ml, ph[t], mem, 0, 0, 0);
      mem = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mh, pl[t], mem, 0, 0, 0);
      mem = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mh, ph[t], mem, 0, 0, 0);
    }
    if (my_row < R) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float x[4], res[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          res[r] = gate * mem[4 * g + r];
          x[r] = ((nan_blocks >> d) & 1u ? NAN : o[d][4 * g + r]) + res[r];
        }
        const size_t at = q_row * IM_D + 32 * d + 8 * g + 4 * half;
        if (a.n_splits == 1)
          *(uint2*)(ro.out + at) = make_uint2((uint32_t)f2bf_rne(x[0]) | ((uint32_t)f2bf_rne(x[1]) << 16),
                                              (uint32_t)f2bf_rne(x[2]) | ((uint32_t)f2bf_rne(x[3]) << 16));
        if (ro.readout) *(float4*)(ro.readout + at) = make_float4(res[0], res[1], res[2], res[3]);
      }
    }
  }
}

// The splits of many rows joined, their readouts (res) added: 2 rows a workgroup of 256.  1024 rows of 32 splits (17 MB): 7.4 us.  (As k_packed_combine, which makes the readout of a
// few rows: 46 us for 8192 rows of 8 splits, 85 us for 16384 of 4.)
__global__ __launch_bounds__(256) void k_packed_join(const float* __restrict__ part, int n_splits, long long rows, const float* __restrict__ res,
                                                     bf16_t* __restrict__ out, float* __restrict__ readout_dbg) {
  const long long row = 2ll * blockIdx.x + (threadIdx.x >> 7);
  const int x = threadIdx.x & 127;
  if (row >= rows) return;
  const float* rec = part + row * n_splits * PG_REC;
  const float r = res[row * IM_D + x];
  float m = PG_NO_MAX, l = 0.f, o = 0.f;
  for (int c0 = 0; c0 < n_splits; c0 += 8) {   // 8 splits at a time
    float cm[8], cl[8], co[8], top = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float* p = rec + (size_t)min(c0 + j, n_splits - 1) * PG_REC;
      cm[j] = p[0]; cl[j] = p[1]; co[j] = p[2 + x];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 + j < n_splits) top = fmaxf(top, cm[j]);
    const float f = __builtin_amdgcn_exp2f(m - top);
    l *= f; o *= f; m = top;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (c0 + j < n_splits) {
        const float e = __builtin_amdgcn_exp2f(cm[j] - m);
        l = fmaf(e, cl[j], l);
        o = fmaf(e, co[j], o);
      }
    }
  }
  out[row * IM_D + x] = f2bf_rne((l == 0.f ? 0.f : o / l) + r);   // (no entry seen: 0)
  if (readout_dbg) readout_dbg[row * IM_D + x] = r;
}

// ------------------------------------------------------------------------------------------
// compaction
// ------------------------------------------------------------------------------------------
// number of entries of the ascending list [0, n) that are below x; for a whole wave: 64 probes a round, 2 rounds for 4096 entries
__device__ __forceinline__ int pg_below(const int32_t* __restrict__ list, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;   // the answer is in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;   // (at is ascending: the lanes whose entry is below x come first)
    const int c = __popcll(__ballot(at < hi && list[at] < x));
    if (c == 0) return lo;
    hi = min(hi, lo + c * step);
    lo += (c - 1) * step + 1;
  }
  return lo;
}

// The plan.  A shared page that has a hole below n_keep is copied (a new page is taken for it, in order, as at an append); pages behind
// n_keep are given up.  The table as it was stays in the scratch for the launch that moves the rows.
__device__ __forceinline__ bool pg_lists_fit(int n, int nk, int ne, int max_live) { return n <= max_live && nk >= 0 && ne >= 0 && nk <= n && nk + ne == n; }

// The plan of a small table, one launch of one workgroup, its notes in LDS (in the workspace a step is a round trip more each): 5 us for 1056
// (unit, page) pairs without shared pages, 10 to 12 with, 16 for 3100.  The three launches of a larger table take 14 to 15 up to 16384 pairs, 31 for
// 32768 with 32000 copies; one workgroup for those: 25 to 60, and 187.
#define PG_PLAN_ITEMS 4096
#define PG_PLAN_UNITS 1024
__global__ __launch_bounds__(1024) void k_packed_plan_compact(int32_t* __restrict__ table, int32_t* __restrict__ refs, int n_pages,
                                                              const int32_t* __restrict__ len, const int32_t* __restrict__ evict_idx,
                                                              const int32_t* __restrict__ n_keep, const int32_t* __restrict__ n_evict,
                                                              int units, int T, int C, int max_live, PgScratch ws,
                                                              int32_t* __restrict__ status) {
  __shared__ int s_wave[16], s_shared, s_rank[PG_PLAN_ITEMS], s_hole[PG_PLAN_ITEMS], s_end[PG_PLAN_UNITS];
  const uint32_t tid = threadIdx.x, lane = tid & 63, items = (uint32_t)units * (uint32_t)T;
  auto lists_fit = [&](int u) { return pg_lists_fit(len[u], n_keep[u], n_evict[u], max_live); };
  if (tid == 0) s_shared = 0;
  __syncthreads();
#pragma unroll 2
  for (uint32_t i = tid; i < items; i += 1024) {
    const uint32_t u = i / (uint32_t)T, p = i - u * T;
    const int page = table[i], nk = n_keep[u], ne = n_evict[u];
    const bool shared = lists_fit(u) && ne > 0 && (int)p * PG_SLOTS < nk && pg_is_page(page, n_pages) && refs[page] > 1;
    ws.old[i] = page;
    s_rank[i] = shared ? 1 : 0;
    s_hole[i] = 0;
    if (shared) s_shared = 1;
  }
  __syncthreads();
  int found = 0;
  const bool any_shared = s_shared != 0;
  if (any_shared) {
#pragma unroll 2
    for (int u = tid >> 6; u < units; u += 16) {
      const int nk = n_keep[u], ne = n_evict[u];
      const int32_t* evict = evict_idx + (size_t)u * C;
      if (!lists_fit(u)) continue;
      bool more = true;
      for (int e0 = 0; e0 < ne && more; e0 += 1024) {
        int e[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) e[j] = e0 + 64 * j + (int)lane < ne ? evict[e0 + 64 * j + lane] : nk;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if ((uint32_t)e[j] < (uint32_t)nk) s_hole[u * T + e[j] / PG_SLOTS] = 1;
        more = !__any(e[15] >= nk);
      }
    }
    __syncthreads();
    int want = 0;
    for (uint32_t i0 = 0; i0 < items; i0 += 1024) {
      const uint32_t i = i0 + tid;
      const int need = i < items ? s_rank[i] & s_hole[i] : 0;
      int total;
      const int before = pg_scan(need, s_wave, total);
      if (i < items) {
        s_rank[i] = need ? want + before : -1;
        if (i % (uint32_t)T == (uint32_t)T - 1) s_end[i / (uint32_t)T] = want + before + need;
      }
      want += total;
    }
    __syncthreads();
    found = want ? pg_find_free(refs, n_pages, want, ws.free_ids, s_wave) : 0;
    __syncthreads();
  }
  auto enough = [&](int u) {
    if (!any_shared) return true;
    const int e = s_end[u], begin = u ? s_end[u - 1] : 0;
    return e == begin || e <= found;
  };
  for (int u = tid; u < units; u += 1024) {
    const bool fit = lists_fit(u), pages = enough(u);
    if (!fit) atomicOr(status, len[u] > max_live ? IM_STATUS_LIVE_EXCEEDED_BIT : IM_STATUS_BAD_LISTS_BIT);
    else if (!pages) atomicOr(status, IM_STATUS_OUT_OF_PAGES_BIT);
    ws.base[u] = fit && pages;
  }
#pragma unroll 2
  for (uint32_t i = tid; i < items; i += 1024) {
    const uint32_t u = i / (uint32_t)T, p = i - u * T;
    const int old = ws.old[i], r = any_shared ? s_rank[i] : -1, nk = n_keep[u];
    const bool fit = lists_fit(u) && enough(u);
    if (old == -1 || !fit) continue;
    if (r >= 0) {
      const int id = ws.free_ids[r];
      table[i] = id;
      refs[id] = 1;
      atomicSub(&refs[old], 1);
    } else if ((int)p * PG_SLOTS >= nk) {
      table[i] = -1;
      if (pg_is_page(old, n_pages)) atomicSub(&refs[old], 1);
    }
  }
}

// The plan of a larger table, three launches.  A workgroup per unit: the table as it was, and which of its pages are to be copied (rank
// among the unit's, -1: not); ws.end[u]: how many they are.
__global__ __launch_bounds__(1024) void k_packed_plan_units(const int32_t* __restrict__ table, const int32_t* __restrict__ refs, int n_pages,
                                                            const int32_t* __restrict__ len, const int32_t* __restrict__ evict_idx,
                                                            const int32_t* __restrict__ n_keep, const int32_t* __restrict__ n_evict, int T,
                                                            int C, int max_live, PgScratch ws) {
  __shared__ int s_wave[16], s_shared;
  const int u = blockIdx.x, tid = threadIdx.x, nk = n_keep[u], ne = n_evict[u];
  const bool fit = pg_lists_fit(len[u], nk, ne, max_live);
  int32_t *old = ws.old + (size_t)u * T, *rank = ws.rank + (size_t)u * T, *hole = ws.free_ids + (size_t)u * T;   // (until there are ids)
  if (tid == 0) s_shared = 0;
  __syncthreads();
#pragma unroll 2
  for (int p = tid; p < T; p += 1024) {
    const int page = table[(size_t)u * T + p];
    const bool shared = fit && ne > 0 && p * PG_SLOTS < nk && pg_is_page(page, n_pages) && refs[page] > 1;
    old[p] = page;
    rank[p] = shared ? 1 : -1;
    hole[p] = 0;
    if (shared) s_shared = 1;
  }
  __syncthreads();
  int want = 0;
  if (s_shared) {
    const int32_t* evict = evict_idx + (size_t)u * C;
    bool more = true;
    for (int e0 = tid; e0 < ne && more; e0 += 8 * 1024) {   // (the list is ascending: behind n_keep there are no more holes)
      int e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = e0 + 1024 * j < ne ? evict[e0 + 1024 * j] : nk;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if ((uint32_t)e[j] < (uint32_t)nk) hole[e[j] / PG_SLOTS] = 1;
      more = e[7] < nk;
    }
    __syncthreads();
    for (int p0 = 0; p0 < T; p0 += 1024) {
      const int p = p0 + tid, need = p < T && rank[p] > 0 && hole[p];
      int total;
      const int before = pg_scan(need, s_wave, total);
      if (p < T) rank[p] = need ? want + before : -1;
      want += total;
    }
  }
  if (tid == 0) ws.end[u] = want;
}

// One workgroup: the units' counts become ends, free pages are looked for, and units that get theirs (base) are told from the others.
__global__ __launch_bounds__(1024) void k_packed_plan_pages(const int32_t* __restrict__ refs, int n_pages, const int32_t* __restrict__ len,
                                                            const int32_t* __restrict__ n_keep, const int32_t* __restrict__ n_evict,
                                                            int units, int max_live, PgScratch ws, int32_t* __restrict__ status) {
  __shared__ int s_wave[16];
  const int tid = threadIdx.x;
  int want = 0;
  for (int u0 = 0; u0 < units; u0 += 1024) {
    const int u = u0 + tid, count = u < units ? ws.end[u] : 0;
    int total;
    const int before = pg_scan(count, s_wave, total);
    if (u < units) ws.end[u] = want + before + count;
    want += total;
  }
  __syncthreads();
  const int found = want ? pg_find_free(refs, n_pages, want, ws.free_ids, s_wave) : 0;
  for (int u = tid; u < units; u += 1024) {
    const int n = len[u], end = ws.end[u], begin = u ? ws.end[u - 1] : 0;
    const bool fit = pg_lists_fit(n, n_keep[u], n_evict[u], max_live), pages = end == begin || end <= found;
    if (!fit) atomicOr(status, n > max_live ? IM_STATUS_LIVE_EXCEEDED_BIT : IM_STATUS_BAD_LISTS_BIT);
    else if (!pages) atomicOr(status, IM_STATUS_OUT_OF_PAGES_BIT);
    ws.base[u] = fit && pages;
  }
}

// grid (ceil(T / 256), units): the table and the counts of users.
__global__ __launch_bounds__(256) void k_packed_plan_table(int32_t* __restrict__ table, int32_t* __restrict__ refs, int n_pages,
                                                           const int32_t* __restrict__ n_keep, int T, PgScratch ws) {
  const int u = blockIdx.y, p = blockIdx.x * 256 + threadIdx.x;
  if (p >= T || !ws.base[u]) return;
  const size_t i = (size_t)u * T + p;
  const int old = ws.old[i], r = ws.rank[i];
  if (r >= 0) {
    const int id = ws.free_ids[(u ? ws.end[u - 1] : 0) + r];
    table[i] = id;
    refs[id] = 1;
    atomicSub(&refs[old], 1);
  } else if (old != -1 && p * PG_SLOTS >= n_keep[u]) {
    table[i] = -1;
    if (pg_is_page(old, n_pages)) atomicSub(&refs[old], 1);
  }
}

// The moves: grid (gx, units), 4 waves.  The first waves move entries, 16 at a time (a row: K 4 lanes of 16 bytes, V 16 words,
// indexer key 8 lanes); the last ones make the copied pages, each from its own rows and those that move into its holes.  Few rows: 6 us, two
// dependent gathers; 128 units with 250 pages each to copy: 102 us, 5.5 TB/s read and written.
__global__ __launch_bounds__(256) void k_packed_compact(char* __restrict__ pages, int n_pages, const int32_t* __restrict__ table, int T,
                                                        bf16_t* __restrict__ Kidx, int32_t* __restrict__ pos, int32_t* __restrict__ len,
                                                        int32_t* __restrict__ n_projected, const int32_t* __restrict__ keep_idx,
                                                        const int32_t* n_keep, const int32_t* __restrict__ evict_idx, int32_t* n_evict, int C, PgScratch ws,
                                                        int32_t* __restrict__ status) {
  const int unit = blockIdx.y, lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6), waves = gridDim.x * 4;
  if (!ws.base[unit]) {   // (a unit that is left as it was has evicted nothing; the plan has read its counts)
    if (blockIdx.x == 0 && threadIdx.x == 0) n_evict[unit] = 0;
    return;
  }
  const int nk = n_keep[unit], ne = n_evict[unit];
  if (blockIdx.x == 0 && threadIdx.x == 0) len[unit] = n_projected[unit] = nk;
  if (ne == 0) return;
  const int32_t *keep = keep_idx + (size_t)unit * C, *evict = evict_idx + (size_t)unit * C;
  const int32_t *old = ws.old + (size_t)unit * T, *tab = table + (size_t)unit * T;
  __shared__ int s_stay;   // kept entries below nk (one wave looks: its probes are 64 cache lines each)
  if (threadIdx.x < 64) {
    const int found = ne < nk ? nk - pg_below(evict, ne, nk) : pg_below(keep, nk, nk);
    if (lane == 0) s_stay = found;
  }
  __syncthreads();
  const int stay = s_stay;
  const int moves = nk - stay;
  // the page that slot s was in; none for a list's entry that is no slot, or a table's that is no page
  auto page_of = [&](int s) {
    const int id = (uint32_t)s < (uint32_t)(nk + ne) ? old[s / PG_SLOTS] : -1;
    return pg_is_page(id, n_pages) ? id : -1;
  };
  auto at_page = [&](int id) { return pages + (size_t)id * PG_BYTES; };
  for (int j0 = 16 * wave; j0 < moves; j0 += 16 * waves) {
    // lane = move (of 16): its slots, the pages they are in; ip: the page to write the row to, none where it is made below
    const bool mine = lane < 16 && j0 + lane < moves;
    const int ss = mine ? keep[stay + j0 + lane] : -1, ds = mine ? evict[j0 + lane] : -1;
    int ps = page_of(ss), pd = (uint32_t)ds < (uint32_t)nk ? tab[ds / PG_SLOTS] : -1;
    if (mine && (ps < 0 || !pg_is_page(pd, n_pages))) {
      atomicOr(status, IM_STATUS_BAD_PAGE_BIT);
      ps = pd = -1;
    }
    const int ip = pd >= 0 && pd == old[ds / PG_SLOTS] ? pd : -1;
    const size_t row0 = (size_t)unit * C;
    uint4 k = {}, ki[2] = {};
    uint32_t v[4] = {}, ks = 0;
    uint8_t vs = 0;
    int at = 0;
    const int rk = lane >> 2, k_ps = __shfl(ps, rk, 64), k_ss = __shfl(ss, rk, 64), k_ip = __shfl(ip, rk, 64), k_ds = __shfl(ds, rk, 64);
    if (k_ip >= 0) {
      k = *(const uint4*)(at_page(k_ps) + 64 * (k_ss % PG_SLOTS) + 16 * (lane & 3));
      vs = (uint8_t)at_page(k_ps)[pg_v_scale(k_ss % PG_SLOTS, lane & 3)];
    }
    int v_ps[4], v_ss[4], v_ip[4], v_ds[4], i_ss[2], i_ds[2];
    bool i_on[2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 4 * t + (lane >> 4);
      v_ps[t] = __shfl(ps, r, 64); v_ss[t] = __shfl(ss, r, 64); v_ip[t] = __shfl(ip, r, 64); v_ds[t] = __shfl(ds, r, 64);
      if (v_ip[t] >= 0) v[t] = *(const uint32_t*)(at_page(v_ps[t]) + pg_v_word(v_ss[t] % PG_SLOTS, lane & 15));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 8 * t + (lane >> 3);
      i_ss[t] = __shfl(ss, r, 64); i_ds[t] = __shfl(ds, r, 64); i_on[t] = __shfl(pd, r, 64) >= 0;
      if (i_on[t]) ki[t] = *(const uint4*)(Kidx + (row0 + i_ss[t]) * IM_DI + 8 * (lane & 7));
    }
    if (pd >= 0) at = pos[row0 + ss];
    if (ip >= 0) ks = *(const uint32_t*)(at_page(ps) + PG_KS + 4 * (ss % PG_SLOTS));
    // (a row that is read here is written by nobody: sources lie at n_keep and above, destinations below)
    if (k_ip >= 0) {
      *(uint4*)(at_page(k_ip) + 64 * (k_ds % PG_SLOTS) + 16 * (lane & 3)) = k;
      at_page(k_ip)[pg_v_scale(k_ds % PG_SLOTS, lane & 3)] = (char)vs;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (v_ip[t] >= 0) *(uint32_t*)(at_page(v_ip[t]) + pg_v_word(v_ds[t] % PG_SLOTS, lane & 15)) = v[t];
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (i_on[t]) *(uint4*)(Kidx + (row0 + i_ds[t]) * IM_DI + 8 * (lane & 7)) = ki[t];
    if (pd >= 0) pos[row0 + ds] = at;
    if (ip >= 0) *(uint32_t*)(at_page(ip) + PG_KS + 4 * (ds % PG_SLOTS)) = ks;
  }
  for (int p = waves - 1 - wave; p * PG_SLOTS < nk; p += waves) {
    if (tab[p] == old[p]) continue;   // (else the plan has taken a page for it)
    // lane = row: where it comes from; holes are evict[first ..] one after another
    const int first = pg_below(evict, ne, p * PG_SLOTS), slot = p * PG_SLOTS + lane;
    const int e = first + lane < moves ? evict[first + lane] - p * PG_SLOTS : -1;   // a hole's row in this page
    unsigned long long holes = 0;
    for (int i = 0; i < 64; ++i) {
      const int r = __builtin_amdgcn_readlane(e, i);
      if ((uint32_t)r >= PG_SLOTS) break;
      holes |= 1ull << r;
    }
    int from = slot < nk ? slot : -1;
    if ((holes >> lane) & 1ull) from = keep[stay + first + __popcll(holes & ((1ull << lane) - 1ull))];
    const int from_page = page_of(from), from_row = from & (PG_SLOTS - 1);
    char* dst = at_page(tab[p]);
    // K: 16 bytes per lane and step, 4 lanes a row; V: words of 4 rows per lane and step
    uint4 k[4];
    uint32_t v[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 16 * t + (lane >> 2), sp = __shfl(from_page, r, 64), sr = __shfl(from_row, r, 64);
      k[t] = make_uint4(0, 0, 0, 0);
      if (sp >= 0) k[t] = *(const uint4*)(at_page(sp) + 64 * sr + 16 * (lane & 3));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rv = 16 * t + 4 * (lane >> 4) + i, vp = __shfl(from_page, rv, 64), vr = __shfl(from_row, rv, 64);
        v[t][i] = 0;
        if (vp >= 0) v[t][i] = *(const uint32_t*)(at_page(vp) + pg_v_word(vr, lane & 15));
      }
    }
    uint32_t ks = 0;
    uint8_t vs[4] = {};
    if (from_page >= 0) {
      ks = *(const uint32_t*)(at_page(from_page) + PG_KS + 4 * from_row);
#pragma unroll
      for (int c = 0; c < 4; ++c) vs[c] = (uint8_t)at_page(from_page)[pg_v_scale(from_row, c)];
    }
    // (rows that come from nowhere lie behind the last kept entry: they may hold anything)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      *(uint4*)(dst + 1024 * t + 16 * lane) = k[t];
      *(uint4*)(dst + PG_V + 1024 * t + 16 * lane) = make_uint4(v[t][0], v[t][1], v[t][2], v[t][3]);
    }
    *(uint32_t*)(dst + PG_KS + 4 * lane) = ks;
#pragma unroll
    for (int c = 0; c < 4; ++c) dst[pg_v_scale(lane, c)] = (char)vs[c];
  }
}

// ------------------------------------------------------------------------------------------
// forks: grid (gx, units), 256 threads
// ------------------------------------------------------------------------------------------
// A sequence that stays is only read, one that changes only written, and counts of users only added to or taken from: no order matters.  Bound by
// the copy of indexer keys, positions and memory: 47 MB read and written 11 us, 4.3 TB/s; the pages' share is their table.
__global__ __launch_bounds__(256) void k_packed_fork(const int32_t* __restrict__ src_of, int32_t* __restrict__ table,
                                                     int32_t* __restrict__ refs, int T, bf16_t* __restrict__ Kidx,
                                                     int32_t* __restrict__ pos, int32_t* __restrict__ len,
                                                     int32_t* __restrict__ n_projected, float* __restrict__ M, float* __restrict__ bvec,
                                                     int n_pages, int B, int H_kv, int C, int32_t* __restrict__ status) {
  const int unit = blockIdx.y, b = unit / H_kv, from = src_of[b];
  if (from == b) return;
  if (from < -1 || from >= B || (from >= 0 && src_of[from] != from)) {
    if (unit % H_kv == 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, IM_STATUS_BAD_FORK_BIT);
    return;
  }
  const int i0 = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256;
  const size_t src = from < 0 ? 0 : (size_t)from * H_kv + unit % H_kv, dst = unit;
  for (int p = i0; p < T; p += step) {
    const int had = table[dst * T + p], gets = from < 0 ? -1 : table[src * T + p];
    if (pg_is_page(gets, n_pages)) atomicAdd(&refs[gets], 1);
    if (pg_is_page(had, n_pages)) atomicSub(&refs[had], 1);
    table[dst * T + p] = gets;
  }
  const int n = from < 0 ? 0 : min(len[src], C);
  for (long long i = i0; i < (long long)n * (IM_DI / 8); i += step)
    ((uint4*)(Kidx + dst * C * IM_DI))[i] = ((const uint4*)(Kidx + src * C * IM_DI))[i];
  for (int i = i0; i < n; i += step) pos[dst * C + i] = pos[src * C + i];
  for (int i = i0; i < IM_DM * IM_D / 4; i += step)
    ((float4*)(M + dst * IM_DM * IM_D))[i] = from < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : ((const float4*)(M + src * IM_DM * IM_D))[i];
  if (blockIdx.x == 0 && threadIdx.x < IM_DM) bvec[dst * IM_DM + threadIdx.x] = from < 0 ? 0.f : bvec[src * IM_DM + threadIdx.x];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    len[dst] = from < 0 ? 0 : len[src];
    n_projected[dst] = from < 0 ? 0 : n_projected[src];
  }
}
