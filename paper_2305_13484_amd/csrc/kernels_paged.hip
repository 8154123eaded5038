// Operators on a cache kept in pages: rows of new tokens into it, their attention over it, the weights that attention gave to its
// rows, and the eviction of the lightest.  A cache is [page][key head][page_size][d]; 16 consecutive positions of a sequence that start
// at a multiple of 16 lie in one page, so whole 16-row groups of a wave share one entry of the page list, which a scalar load fetches.
#include <algorithm>
#include <cmath>

#include "flover_dev.h"
#include "paged.h"

namespace flk {

namespace {

// Lambdas whose captures have to stay in registers.
#define INLINED __attribute__((always_inline))

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What a plan's lists hold is constant while a kernel runs: scalar loads, which no vector load or copy is waited for with.
template <class T> __device__ __forceinline__ T uniform_load(const T* p) {
  struct Words {
    int w[sizeof(T) / 4];
  } x;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) x.w[i] = ((const __attribute__((address_space(4))) int*)(uintptr_t)p)[i];
  return __builtin_bit_cast(T, x);
}

// Row of position pos (uniform in a wave) of a sequence in the cache of one key head.
__device__ __forceinline__ uint32_t cache_row(const PagedView& v, const PagedSeq& s, int kvh, int pos) {
  const int page = quotient(pos, v.by_page);
  return ((uint32_t)uniform_load(v.pages + s.pages + page) * v.n_kv + kvh) * v.page_size + (uint32_t)(pos - page * v.page_size);
}

// ---------------------------------------------------------------- rows of new tokens

// A thread moves 16 bytes of one key head's row of K or V (blockIdx.y); memory bounds it (47 MB read and written in 8.9 us).
__global__ __launch_bounds__(256) void paged_append_kernel(PagedView v, const char* __restrict__ k, int64_t ks, const char* __restrict__ vv,
                                                           int64_t vs, char* __restrict__ kc, char* __restrict__ vc, int row_pieces) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_token = v.n_kv * row_pieces;
  const int t = (int)(i / per_token);
  if (t >= v.tokens) return;
  const int rest = (int)(i - (int64_t)t * per_token), h = rest / row_pieces, piece = rest - h * row_pieces;
  const size_t to = ((size_t)v.places[t] + (size_t)h * v.page_size) * row_pieces + piece;
  if (blockIdx.y == 0) ((u32x4_t*)kc)[to] = *(const u32x4_t*)(k + t * ks + (size_t)rest * 16);
  else ((u32x4_t*)vc)[to] = *(const u32x4_t*)(vv + t * vs + (size_t)rest * 16);
}

// ---------------------------------------------------------------- attention, few rows per key head

// 16 bytes of a cache row.  16-bit caches are read once by the streaming kernel (nothing to keep in the caches); of fp32 ones every 16 query
// rows read them again.
template <int DT> __device__ __forceinline__ u32x4_t load_rows(const char* p) {
  if constexpr (DT == DT_F32) return *(const u32x4_t*)p;
  else return __builtin_nontemporal_load((const u32x4_t*)p);
}

__device__ __forceinline__ f32x4_t mfma_f32(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Two storage elements packed in a dword (or one of fp32) with those that are not finite replaced by zero.
template <int DT> __device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  if constexpr (DT == DT_F32) return (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
  constexpr uint32_t E = DT == DT_F16 ? 0x7c00u : 0x7f80u;
  if ((x & E) == E) x &= 0xffff0000u;
  if ((x & (E << 16)) == (E << 16)) x &= 0xffffu;
  return x;
}
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// permutation of a V row's 16-byte pieces (pairs stay together), so that the keys of a transposing read spread over the banks
template <int D> __device__ __forceinline__ int piece_swizzle(int key) { return D == 128 ? (key & 7) * 2 : ((key >> 1) & 3) * 2; }

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
// Two values rounded to the 16-bit type, to nearest even, in a dword, and the values of its halves.
template <int DT> __device__ __forceinline__ uint32_t round_pair(float a, float b) {
  if constexpr (DT == DT_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), f16x2_t));
}
template <int DT> __device__ __forceinline__ float low_half(uint32_t x) {
  if constexpr (DT == DT_BF16) return __uint_as_float(x << 16);
  else return f16_to_f32((uint16_t)(x & 0xffffu));
}
template <int DT> __device__ __forceinline__ float high_half(uint32_t x) {
  if constexpr (DT == DT_BF16) return __uint_as_float(x & 0xffff0000u);
  else return f16_to_f32((uint16_t)(x >> 16));
}

// Four V^T operands (8 keys of 16 d each) by transposing reads; a[i]: this lane's LDS address of operand i, the second 16 keys lie HI
// bytes further.  Its own wait stands in the block.
template <int HI> __device__ __forceinline__ void read_keys_of_d(const uint32_t (&a)[4], u32x4_t (&v)[4]) {
  uint2 x[4], y[4];
  asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %4, %8 offset:%12\n\t"
               "ds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
               "ds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %6, %10 offset:%12\n\t"
               "ds_read_b64_tr_b16 %3, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
               : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(HI)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = u32x4_t{x[i].x, x[i].y, y[i].x, y[i].y};
}

// One item: 16 query rows of a key head (row r = token r / group of the sequence's new ones, head r % group of the group, so that
// grouped heads share what is read), its four waves taking every fourth step of KT keys; their results are merged through LDS.  The cache is
// read once, straight to registers, the next step's rows on their way while a step is worked on; a token's K and V rows cost 4 operations per
// byte and head of the group, so memory bounds it up to the 16 rows.
//   scores   S^T[key][row] = K . Q^T: a lane's 16 bytes are consecutive d of one key (of one row);
//   softmax  running maximum and sum per row = per output column, 2 in base 2, fp32;
//   output   O^T[d][row] += V^T . P^T: P^T is what the lane holds already; V^T through the wave's own piece of LDS, 16-bit types by
//            transposing reads.  P of 16-bit types enters as two terms, value and rounding remainder (16 bits or more together): memory
//            leaves the time for it.
// Keys that a row does not see have weight zero; if the sum comes out infinite or as no number all the same, it may be such a key's V (0 x inf),
// and the wave's steps are gone through again with those elements kept out of the product and added where they are seen.
// Whole rows go to registers and from there to the wave's LDS, K as well: loading operands straight (16 rows x 64 bytes an instruction, 300 registers,
// one wave per SIMD) read 1.07 GB (64 requests of up to 8192 rows, 32 heads on 8, bf16) in 259 us; this way, two waves per SIMD, in 176 (6.1 TB/s).
template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void paged_rows_kernel(
    PagedView v, const PagedItem* __restrict__ items, const char* __restrict__ q, int64_t qs, const char* __restrict__ kc,
    const char* __restrict__ vc, void* __restrict__ out, float* __restrict__ lse) {
  constexpr int EB = DT == DT_F32 ? 4 : 2, RB = D * EB;       // bytes of an element, of a row
  constexpr int KT = DT == DT_F32 ? 16 : 32, KG = KT / 16;
  constexpr int KS = RB / 64;               // 64-byte steps over a row
  constexpr int LPR = RB / 16, RPI = 64 / LPR, NV = KT / RPI;  // lanes per row, rows per load, loads of a step of K, of V
  constexpr int DTL = D / 16;
  constexpr int LD = D + 4;                 // floats per row of the merge
  constexpr int STEP = KT * RB;             // bytes of a step of K, of V
  __shared__ __attribute__((aligned(1024))) char lds[4][2 * STEP];      // [wave][K | V]
  static_assert(2 * STEP >= 16 * LD * 4, "a wave's results");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int kvh = blockIdx.x % v.n_kv;
  const PagedItem* ip = items + blockIdx.x / v.n_kv;
  const PagedItem it = uniform_load(ip);
  const PagedSeq s = it.s;
  const int rows = s.fresh * v.group;
  const int row = min(it.row0 + n, rows - 1), token = quotient(row, v.by_group), head = kvh * v.group + row - token * v.group;
  const int qpos = s.len - s.fresh + token;                    // sees keys [qlo, qpos] and those below sinks
  const int qlo = v.window > 0 ? qpos - v.window + 1 : 0;
  const int last16 = (s.len - 1) & ~15;

  u32x4_t qf[KS];
  const char* qr = q + (s.first + token) * qs + (size_t)head * RB + g * 16;
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = *(const u32x4_t*)(qr + i * 64);
  const float c = v.scale * kLog2e;

  auto step_key = [&](int u) { return (u < it.gap ? u : u + it.skip) * KT; };
  // rows of a step's 16-key groups in the cache; those behind the last repeat it (hidden below)
  struct Place {
    uint32_t row[KG];
    int most[KG];
  };
  auto place_of = [&](int u, bool first) INLINED {
    Place pl;
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      const int p = min(step_key(u) + kg * 16, last16);
      pl.row[kg] = first ? uniform_load(&ip->place[2 * wave + kg]) + kvh * v.page_size : cache_row(v, s, kvh, p);
      pl.most[kg] = s.len - 1 - p;
    }
    return pl;
  };
  const int lr = lane / LPR, seg = lane % LPR;
  auto load = [&](const Place& pl, u32x4_t(&kr)[NV], u32x4_t(&vr)[NV]) INLINED {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      constexpr int G = 16 / RPI;             // loads of a group
      const size_t at = (size_t)(pl.row[j / G] + min(j % G * RPI + lr, pl.most[j / G])) * RB + seg * 16;
      kr[j] = load_rows<DT>(kc + at);
      vr[j] = load_rows<DT>(vc + at);
    }
  };

  f32x4_t oacc[DTL];
  float m, l;
  char *mk = lds[wave], *mv = lds[wave] + STEP;
  const int vk = 4 * g + (n >> 2);
  const uint32_t vaddr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mv +
                         (uint32_t)((vk * LPR + (((n & 3) >> 1) ^ piece_swizzle<D>(vk))) * 16 + (n & 1) * 8);
  auto k_swizzle = [](int key) { return LPR == 8 ? (key >> 1) & 7 : key & 15; };
  auto v_swizzle = [](int key) { return DT == DT_F32 ? (key >> 2 & 3) * 4 : piece_swizzle<D>(key); };
  auto store = [&](const u32x4_t(&kr)[NV], u32x4_t(&vr)[NV], auto careful) INLINED {
    if constexpr (decltype(careful)::value) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) vr[j][e] = finite_only<DT>(vr[j][e]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int r = j * RPI + lr;
      *(u32x4_t*)(mk + r * RB + (seg ^ k_swizzle(r)) * 16) = kr[j];
      *(u32x4_t*)(mv + r * RB + (seg ^ v_swizzle(r)) * 16) = vr[j];
    }
  };

  auto consume = [&](int u, auto careful) INLINED {
    const int k0 = step_key(u);
    float p[KG * 4], top = -INFINITY;
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      f32x4_t sacc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const u32x4_t kf = *(const u32x4_t*)(mk + (kg * 16 + n) * RB + ((i * 4 + g) ^ k_swizzle(n)) * 16);
        if constexpr (DT == DT_F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc = mfma_f32(__uint_as_float(kf[e]), __uint_as_float(qf[i][e]), sacc);
        } else {
          sacc = mfma16<DT>(kf, qf[i], sacc);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = k0 + kg * 16 + 4 * g + r;
        const bool seen = (key <= qpos) & ((key >= qlo) | (key < v.sinks));
        p[kg * 4 + r] = seen ? sacc[r] * c : -INFINITY;
        top = fmaxf(top, p[kg * 4 + r]);
      }
    }
    top = max_partner<32>(max_partner<16>(top));
    const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.f : mn;
    const float alpha = __builtin_amdgcn_exp2f(m - ms);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int j = 0; j < KG * 4; ++j) {
      p[j] = __builtin_amdgcn_exp2f(p[j] - ms);
      l += p[j];                                               // this lane's share
    }
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt) oacc[dt] *= alpha;
    if constexpr (DT == DT_F32) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int dt = 0; dt < DTL; ++dt)
          oacc[dt] = mfma_f32(*(const float*)(mv + (4 * g + r) * RB + ((dt * 4 + (n >> 2)) ^ (g * 4)) * 16 + (n & 3) * 4), p[r], oacc[dt]);
    } else {
      u32x4_t hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        hi[j] = round_pair<DT>(p[2 * j], p[2 * j + 1]);
        lo[j] = round_pair<DT>(p[2 * j] - low_half<DT>(hi[j]), p[2 * j + 1] - high_half<DT>(hi[j]));
      }
#pragma unroll
      for (int d4 = 0; d4 < DTL; d4 += 4) {
        uint32_t at[4];
        u32x4_t va[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = vaddr ^ ((d4 + i) * 32);
        read_keys_of_d<16 * RB>(at, va);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          oacc[d4 + i] = mfma16<DT>(va[i], lo, oacc[d4 + i]);
          oacc[d4 + i] = mfma16<DT>(va[i], hi, oacc[d4 + i]);
        }
      }
    }
    if constexpr (decltype(careful)::value) {
      for (int j = 0; j < KT; ++j) {
        const int key = k0 + j;
        if (key >= s.len) break;
        const uint32_t r = cache_row(v, s, kvh, key & ~15) + (key & 15);
        const bool seen = (key <= qpos) & ((key >= qlo) | (key < v.sinks));
#pragma unroll
        for (int dt = 0; dt < DTL; ++dt) {
          const f32x4_t x = ldv4<DT>(vc, (size_t)r * D + dt * 16 + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[dt][e] += (seen & !is_finite(x[e])) ? x[e] : 0.f;
        }
      }
    }
  };

  auto all_keys = [&](auto careful) INLINED {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt) oacc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int u = it.u0 + wave;
    if (u < it.u1) {
      u32x4_t kr[NV], vr[NV];
      load(place_of(u, true), kr, vr);
      for (; u + 4 < it.u1; u += 4) {
        const Place next = place_of(u + 4, false);
        store(kr, vr, careful);
        load(next, kr, vr);
        consume(u, careful);
      }
      store(kr, vr, careful);
      consume(u, careful);
    }
    bool fine = true;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) fine &= is_finite(oacc[dt][e]);
    return fine;
  };
  if (!__all(all_keys(std::false_type{}))) all_keys(std::true_type{});

  // the waves' results of a row, in the order of the waves
  l = sum_partner<32>(sum_partner<16>(l));
  __syncthreads();
  float* my = (float*)lds[wave] + n * LD;
#pragma unroll
  for (int dt = 0; dt < DTL; ++dt) *(f32x4_t*)(my + dt * 16 + 4 * g) = oacc[dt];
  if (g == 0) {
    my[D] = m;
    my[D + 1] = l;
  }
  __syncthreads();
  const int r = threadIdx.x >> 4, i = threadIdx.x & 15;
  if (it.row0 + r >= rows) return;
  const float* from = (const float*)lds + r * LD;
  constexpr int W = 2 * STEP / 4;
  const float mt = fmaxf(fmaxf(from[D], from[W + D]), fmaxf(from[2 * W + D], from[3 * W + D])), ms = mt == -INFINITY ? 0.f : mt;
  float lt = 0.f;
  f32x4_t o[D / 64];
#pragma unroll
  for (int e = 0; e < D / 64; ++e) o[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a = __builtin_amdgcn_exp2f(from[w * W + D] - ms);
    lt = fmaf(a, from[w * W + D + 1], lt);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) o[e] += a * ld4(from + w * W + i * (D / 16) + e * 4);
  }
  const int tk = quotient(it.row0 + r, v.by_group), hd = kvh * v.group + it.row0 + r - tk * v.group;
  if (it.part < 0) {
    const size_t at = (size_t)(s.first + tk) * v.n_head + hd;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) stv4<DT>(out, at * D + i * (D / 16) + e * 4, o[e] / lt);
    if (lse && i == 0) lse[at] = mt * kLn2 + logf(lt);
  } else {
    const size_t at = (size_t)it.part + kvh * kRowTile + r;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) *(f32x4_t*)(v.po + at * D + i * (D / 16) + e * 4) = o[e];
    if (i == 0) *(float2*)(v.pm + at * 2) = make_float2(mt, lt);
  }
}

// ---------------------------------------------------------------- attention, many rows per key head

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

// D[32][32] += A[32][16] . B[16][32]: a lane holds row (column) lane % 32 of A (B), 8 consecutive k from 8 * (lane / 32), and of D column lane % 32,
// rows i % 4 + 8 * (i / 4) + 4 * (lane / 32), i < 16
template <int DT> __device__ __forceinline__ f32x16_t mfma32(const u32x4_t& a, const u32x4_t& b, f32x16_t c) {
  if constexpr (DT == DT_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
// V^T operands of twice 16 keys (RB * 16 bytes apart, OFF bytes from a on) and N times 32 d by transposing reads: 16 lanes give the addresses of 4 keys
// x 16 d and get 4 keys of one d each; the second four keys of a lane lie 8 rows further.  The wait stands in the block.
template <int RB, int OFF> __device__ __forceinline__ void read_keys_of_32d(const uint32_t (&a)[4], u32x4_t (&v)[2][4]) {
  uint2 x[16];
  asm volatile("ds_read_b64_tr_b16 %0, %16 offset:%20\n\tds_read_b64_tr_b16 %1, %16 offset:%21\n\t"
               "ds_read_b64_tr_b16 %2, %17 offset:%20\n\tds_read_b64_tr_b16 %3, %17 offset:%21\n\t"
               "ds_read_b64_tr_b16 %4, %18 offset:%20\n\tds_read_b64_tr_b16 %5, %18 offset:%21\n\t"
               "ds_read_b64_tr_b16 %6, %19 offset:%20\n\tds_read_b64_tr_b16 %7, %19 offset:%21\n\t"
               "ds_read_b64_tr_b16 %8, %16 offset:%22\n\tds_read_b64_tr_b16 %9, %16 offset:%23\n\t"
               "ds_read_b64_tr_b16 %10, %17 offset:%22\n\tds_read_b64_tr_b16 %11, %17 offset:%23\n\t"
               "ds_read_b64_tr_b16 %12, %18 offset:%22\n\tds_read_b64_tr_b16 %13, %18 offset:%23\n\t"
               "ds_read_b64_tr_b16 %14, %19 offset:%22\n\tds_read_b64_tr_b16 %15, %19 offset:%23\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]),
                 "=&v"(x[9]), "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
               : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(OFF), "n"(OFF + 8 * RB), "n"(OFF + 16 * RB), "n"(OFF + 24 * RB)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = u32x4_t{x[2 * i].x, x[2 * i].y, x[2 * i + 1].x, x[2 * i + 1].y};
}
template <int RB, int OFF> __device__ __forceinline__ void read_keys_of_32d(const uint32_t (&a)[2], u32x4_t (&v)[2][2]) {
  uint2 x[8];
  asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %8 offset:%11\n\t"
               "ds_read_b64_tr_b16 %2, %9 offset:%10\n\tds_read_b64_tr_b16 %3, %9 offset:%11\n\t"
               "ds_read_b64_tr_b16 %4, %8 offset:%12\n\tds_read_b64_tr_b16 %5, %8 offset:%13\n\t"
               "ds_read_b64_tr_b16 %6, %9 offset:%12\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
               : "v"(a[0]), "v"(a[1]), "n"(OFF), "n"(OFF + 8 * RB), "n"(OFF + 16 * RB), "n"(OFF + 24 * RB)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i / 2][i % 2] = u32x4_t{x[2 * i].x, x[2 * i].y, x[2 * i + 1].x, x[2 * i + 1].y};
}

// 16 bytes of LDS from each of N addresses, OFF bytes further, with their wait: at an LDS read of its own the compiler waits for every
// asynchronous copy in flight.
template <int OFF> __device__ __forceinline__ void read_pieces(const uint32_t (&a)[4], u32x4_t (&v)[4]) {
  asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\tds_read_b128 %2, %6 offset:%8\n\t"
               "ds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
               : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(OFF)
               : "memory");
}
template <int OFF> __device__ __forceinline__ void read_pieces(const uint32_t (&a)[8], u32x4_t (&v)[8]) {
  asm volatile("ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%16\n\tds_read_b128 %2, %10 offset:%16\n\t"
               "ds_read_b128 %3, %11 offset:%16\n\tds_read_b128 %4, %12 offset:%16\n\tds_read_b128 %5, %13 offset:%16\n\t"
               "ds_read_b128 %6, %14 offset:%16\n\tds_read_b128 %7, %15 offset:%16\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
               : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "n"(OFF)
               : "memory");
}

// One item of 128 query rows of a key head, 32 per wave; the block's waves share the keys, 64 at a time, the next 64 rows of K and V on their way
// to LDS (asynchronous copies, two buffers) while the present ones are worked on.  16-bit types.
//   scores   S^T[key][row] = K . Q^T in tiles of 32 x 32, so that a row's scores lie in two lanes;
//   softmax  running maximum and sum per row in fp32.  The maximum follows only when a score passes it by 8 (in base 2): weights are up to
//            2^8 then, and the sums are scaled again rarely;
//   output   O^T[d][row] += V^T . P^T: P^T is what the lanes hold, rounded to the 16-bit type (half a step of the weight, like the
//            output's own rounding; the sum in the denominator is of the unrounded ones); V^T by transposing reads.
// LDS rows are the cache's, their 16-byte pieces permuted by key so that a read's keys spread over the banks.  Steps that every row of the wave
// sees in full take no mask.  A sum that is infinite or no number: as in paged_rows_kernel, the block goes through its keys again.
// Per step and wave the matrix unit has 1024 cycles (d = 128), the vector unit about 900 (32 exponentials of 16 cycles each, and the maximum, the
// scaling, the sum, the rounding of 32 scores), the compute unit's LDS 256; two waves of different blocks share a SIMD, and one that has its scores
// goes first.  2 x 2048 tokens over 7000 and 8192 rows, 32 heads on 8, bf16: 420 to 436 us, 1.01 to 1.05 PFLOP/s (without that priority 3 % more; with LDS reads that
// the compiler waits for copies at 567; 16 rows per block 3680).
template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void paged_tile_kernel(
    PagedView v, const PagedItem* __restrict__ items, const char* __restrict__ q, int64_t qs, const char* __restrict__ kc,
    const char* __restrict__ vc, void* __restrict__ out, float* __restrict__ lse) {
  constexpr int RB = D * 2, KS = D / 16, DTL = D / 32, SEG = D / 8;      // row bytes, 16-d steps, 32-d tiles, 16-byte pieces of a row
  constexpr int RPC = 64 / SEG, NC = 16 / RPC;                          // rows of a copy, copies of 16 rows
  constexpr int BUF = kTileKeys * RB;
  __shared__ __attribute__((aligned(1024))) char lds[2][2][BUF];        // [buffer][K | V]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, n = lane & 31;
  const int kvh = blockIdx.x % v.n_kv;
  const PagedItem* ip = items + blockIdx.x / v.n_kv;
  const PagedItem it = uniform_load(ip);
  const PagedSeq s = it.s;
  const int rows = s.fresh * v.group, before = s.len - s.fresh;
  const int row0 = it.row0 + wave * 32;
  const int row = min(row0 + n, rows - 1), token = quotient(row, v.by_group), head = kvh * v.group + row - token * v.group;
  const int qpos = before + token, qlo = v.window > 0 ? qpos - v.window + 1 : 0;
  // positions of the wave's rows: [p0, p1]
  const int p0 = before + quotient(min(row0, rows - 1), v.by_group), p1 = row0 < rows ? before + quotient(min(row0 + 31, rows - 1), v.by_group) : -1;
  const int last16 = (s.len - 1) & ~15;
  u32x4_t qf[KS];
  const char* qr = q + (s.first + token) * qs + (size_t)head * RB + h * 16;
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = *(const u32x4_t*)(qr + i * 32);
  const float c = v.scale * kLog2e;

  auto step_key = [&](int u) { return (u < it.gap ? u : u + it.skip) * kTileKeys; };
  // a wave copies rows 16 * wave .. + 15 of a step; rows behind the last repeat it (hidden below)
  auto place_of = [&](int u) INLINED { return min(step_key(u) + wave * 16, last16); };
  auto k_swizzle = [](int key) { return D == 128 ? key & 15 : (key >> 1) & 7; };
  // 32 lanes of a transposing read take 64 bytes of each of four keys: their pieces lie on four quarters of the banks (with piece_swizzle a third of the
  // LDS cycles were conflicts; the time is the same within 1 %)
  auto v_swizzle = [](int key) { return (D == 128 ? key & 3 : key >> 1 & 1) * 4; };
  auto issue = [&](int u, uint32_t r0) INLINED {
    char(*buf)[BUF] = lds[(u - it.u0) & 1];
    const int most = s.len - 1 - place_of(u);
    const char *kb = kc + (size_t)r0 * RB, *vb = vc + (size_t)r0 * RB;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int r = j * RPC + lane / SEG, key = wave * 16 + r, from = min(r, most) * RB;
      copy_to_lds(kb, from + ((lane % SEG) ^ k_swizzle(key)) * 16, (u32x4_t*)(buf[0] + wave * 16 * RB + j * 1024));
      copy_to_lds(vb, from + ((lane % SEG) ^ v_swizzle(key)) * 16, (u32x4_t*)(buf[1] + wave * 16 * RB + j * 1024));
    }
  };
  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0][0];
  // this lane's 8 bytes of V for the first operand: key 4h + i / 4, d 16 * (second 16 lanes) + 4 * (i % 4), i = lane % 16
  const int vk = 4 * h + ((lane & 15) >> 2), vp = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const uint32_t kaddr = lds_at + (uint32_t)(n * RB + (h ^ k_swizzle(n)) * 16);
  const uint32_t vaddr = lds_at + BUF + (uint32_t)(vk * RB + (vp ^ v_swizzle(vk)) * 16 + (lane & 1) * 8);

  f32x16_t oacc[DTL];
  float m, l;                                 // the running maximum (of unscaled scores), this lane's share of the sum
  auto consume = [&](int u, auto careful_) INLINED {
    constexpr bool careful = decltype(careful_)::value;
    const int k0 = step_key(u), b = (u - it.u0) & 1;
    if (k0 > p1) return;                      // none of the wave's rows sees these keys
    const bool full = k0 + kTileKeys - 1 <= p0 && (v.window <= 0 || k0 > p1 - v.window || k0 + kTileKeys <= v.sinks);
    f32x16_t sacc[2];
    uint32_t ka[KS];
    u32x4_t kf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ka[ks] = (kaddr + b * (2 * BUF)) ^ (ks * 32);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sacc[kt][i] = 0.f;
      if (kt == 0) read_pieces<0>(ka, kf);
      else read_pieces<32 * RB>(ka, kf);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sacc[kt] = mfma32<DT>(kf[ks], qf[ks], sacc[kt]);
    }
    u32x4_t va[2][2][DTL];                    // 16-key steps; on their way while the products are worked on
    uint32_t at[DTL];
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt) at[dt] = (vaddr + b * (2 * BUF)) ^ (dt * 64);
    read_keys_of_32d<RB, 0>(at, va[0]);
    read_keys_of_32d<RB, 32 * RB>(at, va[1]);
    if (careful || !full) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = k0 + kt * 32 + (i & 3) + 8 * (i >> 2) + 4 * h;
          sacc[kt][i] = ((key <= qpos) & ((key >= qlo) | (key < v.sinks))) ? sacc[kt][i] : -INFINITY;
        }
    }
    __builtin_amdgcn_s_setprio(1);
    float top = sacc[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, sacc[i >> 4][i & 15]);
    top = max_partner<32>(top);
    if (__any((top - m) * c > 8.f)) {          // (a first maximum passes minus infinity by infinity)
      const float mn = fmaxf(m, top);
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * c);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < DTL; ++dt) oacc[dt] *= alpha;
    }
    const float mc = m == -INFINITY ? 0.f : m * c;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sacc[i >> 4][i & 15], c, -mc));
      sacc[i >> 4][i & 15] = p;
      l += p;
    }
#pragma unroll
    for (int st = 0; st < 4; ++st) {           // 16 keys
      u32x4_t pb;
#pragma unroll
      for (int e = 0; e < 4; ++e) pb[e] = round_pair<DT>(sacc[st >> 1][(st & 1) * 8 + 2 * e], sacc[st >> 1][(st & 1) * 8 + 2 * e + 1]);
#pragma unroll
      for (int dt = 0; dt < DTL; ++dt) {
        if constexpr (careful) {
#pragma unroll
          for (int e = 0; e < 4; ++e) va[st >> 1][st & 1][dt][e] = finite_only<DT>(va[st >> 1][st & 1][dt][e]);
        }
        oacc[dt] = mfma32<DT>(va[st >> 1][st & 1][dt], pb, oacc[dt]);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (careful) {
      for (int j = 0; j < kTileKeys; ++j) {
        const int key = k0 + j;
        if (key >= s.len) break;
        const uint32_t r = cache_row(v, s, kvh, key & ~15) + (key & 15);
        const bool seen = (key <= qpos) & ((key >= qlo) | (key < v.sinks));
#pragma unroll
        for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const f32x4_t x = ldv4<DT>(vc, (size_t)r * D + dt * 32 + 2 * i + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[dt][i + e] += (seen & !is_finite(x[e])) ? x[e] : 0.f;
          }
      }
    }
  };
  auto all_keys = [&](auto careful) INLINED {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
    issue(it.u0, uniform_load(&ip->place[wave]) + kvh * v.page_size);
    uint32_t next = it.u0 + 1 < it.u1 ? cache_row(v, s, kvh, place_of(it.u0 + 1)) : 0;
    for (int u = it.u0; u < it.u1; ++u) {
      copies_barrier<0>(true);                 // step u has landed; every wave is done with step u - 1
      if (u + 1 < it.u1) issue(u + 1, next);
      if (u + 2 < it.u1) next = cache_row(v, s, kvh, place_of(u + 2));
      consume(u, careful);
    }
    bool fine = true;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) fine &= is_finite(oacc[dt][i]);
    return fine;
  };
  if (__syncthreads_or(!all_keys(std::false_type{}))) all_keys(std::true_type{});      // (behind the barrier the buffers are free)

  l = sum_partner<32>(l);
  if (row0 + n >= rows) return;
  const int tk = quotient(row0 + n, v.by_group);
  if (it.part < 0) {
    const size_t at = (size_t)(s.first + tk) * v.n_head + kvh * v.group + row0 + n - tk * v.group;
    const float inv = 1.f / l;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        stv4<DT>(out, at * D + dt * 32 + 2 * i + 4 * h,
                 f32x4_t{oacc[dt][i] * inv, oacc[dt][i + 1] * inv, oacc[dt][i + 2] * inv, oacc[dt][i + 3] * inv});
    if (lse && h == 0) lse[at] = m * v.scale + logf(l);
  } else {
    const size_t at = (size_t)it.part + kvh * kTileRows + wave * 32 + n;
#pragma unroll
    for (int dt = 0; dt < DTL; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4_t*)(v.po + at * D + dt * 32 + 2 * i + 4 * h) = f32x4_t{oacc[dt][i], oacc[dt][i + 1], oacc[dt][i + 2], oacc[dt][i + 3]};
    if (h == 0) *(float2*)(v.pm + at * 2) = make_float2(m * c, l);
  }
}

// Rows whose keys went to several items.  W waves per row, 4 / W rows per block; D / 4 lanes hold a row, and every group of so many lanes takes
// its share of the parts, in order; the groups' results are joined in their order.  Few blocks have all the parts of a single long sequence to
// read: four waves per row then (one row of 64 parts: 32 KB).
template <int DT, int D, int W>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedView v, const PagedMerge* __restrict__ merges, void* __restrict__ out,
                                                          float* __restrict__ lse) {
  constexpr int LPR = D / 4, GR = 64 * W / LPR, ROWS = 4 / W;
  __shared__ __attribute__((aligned(16))) float part[ROWS][GR][D + 4];
  const int kvh = blockIdx.x % v.n_kv;
  const PagedMerge mg = uniform_load(merges + blockIdx.x / v.n_kv);
  const PagedSeq s = mg.s;
  const int which = threadIdx.x / (64 * W), r = blockIdx.y * ROWS + which;
  const int grp = threadIdx.x % (64 * W) / LPR, i = threadIdx.x % LPR * 4;
  const int rows = min(16, s.fresh * v.group - mg.row0);
  if (blockIdx.y * ROWS >= rows) return;                       // the whole block
  const size_t first = (size_t)mg.part + kvh * mg.tile + min(r, rows - 1), stride = mg.stride;
  float m = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = grp; p0 < mg.parts; p0 += 4 * GR) {
    float2 ml[4];
    f32x4_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t at = first + (size_t)min(p0 + j * GR, mg.parts - 1) * stride;
      ml[j] = *(const float2*)(v.pm + at * 2);
      x[j] = ld4(v.po + at * D + i);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p0 + j * GR < mg.parts) {
        const float mn = fmaxf(m, ml[j].x), ms = mn == -INFINITY ? 0.f : mn;
        const float a = __builtin_amdgcn_exp2f(m - ms), b = __builtin_amdgcn_exp2f(ml[j].x - ms);
        l = fmaf(b, ml[j].y, a * l);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(b, x[j][e], a * o[e]);
        m = mn;
      }
  }
  float* mine = part[which][grp];
  *(f32x4_t*)(mine + i) = o;
  if (i == 0) {
    mine[D] = m;
    mine[D + 1] = l;
  }
  __syncthreads();
  if (grp > 0 || r >= rows) return;
  float mt = -INFINITY;
#pragma unroll
  for (int g = 0; g < GR; ++g) mt = fmaxf(mt, part[which][g][D]);
  const float ms = mt == -INFINITY ? 0.f : mt;
  float lt = 0.f;
  o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const float a = __builtin_amdgcn_exp2f(part[which][g][D] - ms);
    lt = fmaf(a, part[which][g][D + 1], lt);
    const f32x4_t x = ld4(&part[which][g][i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(a, x[e], o[e]);
  }
  const int tk = quotient(mg.row0 + r, v.by_group), hd = kvh * v.group + mg.row0 + r - tk * v.group;
  const size_t at = (size_t)(s.first + tk) * v.n_head + hd;
  stv4<DT>(out, at * D + i, o / lt);
  if (lse && i == 0) lse[at] = mt * kLn2 + logf(lt);
}

// ---------------------------------------------------------------- weights that the new tokens gave to the cached rows

__device__ __forceinline__ void copy_words_to_lds(const char* base, uint32_t off, float* l) {      // 64 lanes x 4 bytes, as copy_to_lds
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, -1, 0x00020000),
                                           (__attribute__((address_space(3))) void*)l, 4, off, 0, 0, 0);
}
// Whether a sequence's weights are the streaming kernel's, or the tile kernel's.
__device__ __forceinline__ bool few_rows(int rows) { return rows <= kRowTile; }
// New tokens [t0, t1) of a sequence see some of keys [k0, k1).
__device__ __forceinline__ int first_token(const PagedSeq& s, int k0) { return max(0, k0 - (s.len - s.fresh)); }
__device__ __forceinline__ int end_token(const PagedView& v, const PagedSeq& s, int k0, int k1) {
  return v.window > 0 && k0 >= v.sinks ? min(s.fresh, k1 - 1 + v.window - (s.len - s.fresh)) : s.fresh;
}
// The new weight of position key: rows that the new tokens brought begin with none.
__device__ __forceinline__ float new_weight(float given, float old, float decay, bool brought) {
  return decay == 0.f || brought ? given : fmaf(decay, old, given);
}

// grid = (blocks of `keys` positions, n_kv, n_seq).  Few rows of queries: K streams through as in paged_rows_kernel (a wave takes every
// fourth step, whole rows to registers, to the wave's piece of LDS, from there as operands) and bounds it.  S[row][key] = Q . K^T leaves a key's
// scores in one column, so that their exponentials add up in a lane.  64 requests of 4096 rows, 8 key heads, bf16: 92 us (5.8 TB/s).
template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DT == DT_F32 ? 2 : 4))) void paged_weights_rows_kernel(
    PagedView v, const char* __restrict__ q, int64_t qs, const char* __restrict__ kc, const float* __restrict__ lse, float decay,
    float* __restrict__ w, int64_t ws, int keys) {
  constexpr int EB = DT == DT_F32 ? 4 : 2, RB = D * EB, KS = RB / 64;
  constexpr int KT = DT == DT_F32 ? 16 : 32, KG = KT / 16, LPR = RB / 16, RPI = 64 / LPR, NV = KT / RPI;
  __shared__ __attribute__((aligned(1024))) char lds[4][KT * RB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, n = lane & 15, kvh = blockIdx.y;
  const PagedSeq s = uniform_load(v.seqs + blockIdx.z);
  if (!few_rows(s.fresh * v.group)) return;
  const int before = s.len - s.fresh, last16 = (s.len - 1) & ~15;
  const int end = min(s.len, (int)(blockIdx.x + 1) * keys);
  int k0 = blockIdx.x * keys + wave * KT;
  if (k0 >= end) return;
  const float c = v.scale * kLog2e;
  char* mk = lds[wave];
  auto k_swizzle = [](int key) { return LPR == 8 ? (key >> 1) & 7 : key & 15; };
  u32x4_t kr[NV];
  const int lr = lane / LPR, seg = lane % LPR;
  auto load = [&](int k) INLINED {
    uint32_t row[KG];
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) row[kg] = cache_row(v, s, kvh, min(k + kg * 16, last16));
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      constexpr int G = 16 / RPI;
      const int most = s.len - 1 - min(k + j / G * 16, last16);
      kr[j] = load_rows<DT>(kc + (size_t)(row[j / G] + min(j % G * RPI + lr, most)) * RB + seg * 16);
    }
  };
  u32x4_t qf[KS];
  float base[4];                                               // of rows 4g + r: lse in base 2, and the position
  int at[4];
  const int rows = s.fresh * v.group;
  auto queries = [&]() INLINED {
    const int row = min(n, rows - 1), token = quotient(row, v.by_group), head = kvh * v.group + row - token * v.group;
    const char* qr = q + (s.first + token) * qs + (size_t)head * RB + g * 16;
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[i] = *(const u32x4_t*)(qr + i * 64);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int rr = min(4 * g + r, rows - 1), tk = quotient(rr, v.by_group);
      base[r] = lse[(size_t)(s.first + tk) * v.n_head + kvh * v.group + rr - tk * v.group] * kLog2e;
      at[r] = 4 * g + r < rows ? before + tk : -1;             // -1: no such row
    }
  };
  auto seen = [&](int k) INLINED { return first_token(s, k) < end_token(v, s, k, min(k + KT, s.len)); };      // by some new token
  if (seen(k0)) load(k0);
  if (rows > 0) queries();
  for (; k0 < end; k0 += 4 * KT) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int r = j * RPI + lr;
      *(u32x4_t*)(mk + r * RB + (seg ^ k_swizzle(r)) * 16) = kr[j];
    }
    // the lane that holds a key's sum at the end: group kg of the lanes key group kg
    const int mine = k0 + g * 16 + n;
    float* to = w + ((int64_t)blockIdx.z * v.n_kv + kvh) * ws + mine;
    const bool writes = g < KG && mine < s.len, brought = mine >= before;
    const float old = writes && decay != 0.f && !brought ? *to : 0.f;
    if (k0 + 4 * KT < end && seen(k0 + 4 * KT)) load(k0 + 4 * KT);
    float sum[KG];
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) sum[kg] = 0.f;
    if (seen(k0)) {
#pragma unroll
      for (int kg = 0; kg < KG; ++kg) {
        f32x4_t sacc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const u32x4_t kf = *(const u32x4_t*)(mk + (kg * 16 + n) * RB + ((i * 4 + g) ^ k_swizzle(n)) * 16);
          if constexpr (DT == DT_F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sacc = mfma_f32(__uint_as_float(qf[i][e]), __uint_as_float(kf[e]), sacc);
          } else {
            sacc = mfma16<DT>(qf[i], kf, sacc);
          }
        }
        const int key = k0 + kg * 16 + n;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool seen = (key <= at[r]) & ((v.window <= 0) | (key > at[r] - v.window) | (key < v.sinks));
          sum[kg] += __builtin_amdgcn_exp2f(seen ? fmaf(sacc[r], c, -base[r]) : -INFINITY);
        }
      }
    }
    float t = 0.f;
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      const float x = sum_partner<32>(sum_partner<16>(sum[kg]));
      t = g == kg ? x : t;
    }
    if (writes) *to = new_weight(t, old, decay, brought);
  }
}

// Many rows of queries.  A wave holds the K rows of 32 positions as operands and goes through the rows of queries that see any of them; S[row][key]
// as above, a lane adds up the rows of its key (fp32: two keys, of either 16-key group).  The rows come to LDS by asynchronous copies, a ring of steps.
//   SPLIT = false: grid = n_kv x entries of 128 positions, the four waves share steps of 64 rows (fp32: 32), three in the ring;
//   SPLIT = true:  grid = (n_kv x entries, 4), 32 positions, every wave has its own steps of half as many rows, each fourth one, two in the ring,
//                  and the waves' sums are joined in their order: four times the blocks and a quarter of the rows each, for four times the rows read.
// Split where blocks of 128 positions are 128 or fewer, one for two compute units (us, shared -> split, d = 128: 64 blocks, 8 heads, 100 new tokens of
// 1000 rows 6.2 -> 5.0, 32 heads on 8, 1000 of 1000 64 -> 27; 128 blocks, 200 of 2000 18.8 -> 12.4, 2000 of 2000 122 -> 90; 192 blocks, 16 heads,
// 1500 of 1500 28.1 -> 24.2, 500 of 1500 13.4 -> 16.2; 256 blocks, 32 heads, 1000 of 1000 20.9 -> 26.9).
// 16-bit types: vector instructions bound it, an exponential takes 16 cycles of a wave, its product's share 8, the sum and the scaling 4 each.  fp32:
// the products (16 x 16 x 4).  2048 new tokens of 8192 rows, 32 heads on 8, bf16: 180 us; 1000 of 3000, fp32: 315.

// The rows of a block's, or of a wave's, steps and their lse.
template <int RB, int ROWS, int WAVES, int RING> struct QueryRing {
  static constexpr int SEG = RB / 16, RPC = 64 / SEG, NC = ROWS / WAVES / RPC;      // pieces of a row, rows of a copy, copies of a wave per step
  char* rows;                     // LDS: [RING][ROWS * RB], 16-byte pieces permuted by row
  float* lse;                     // LDS: [RING][64], of every wave for itself
  const char* q;
  const float* from_lse;
  int64_t qs;
  int b0, b1, wave, lane, kvh;    // rows [b0, b1) of the sequence; the wave among those that share the steps
  uint32_t at[NC], lse_at;        // offsets of the lane's pieces of a step from the step's first token on
  bool alike;                     // steps begin with a token: the same offsets, but for the last
  static __device__ __forceinline__ int swizzle(int row) { return SEG == 8 ? (row >> 1) & 7 : row & 15; }
  __device__ __forceinline__ void start(const PagedView& v, const PagedSeq& s, const char* q_, int64_t qs_, const float* lse_, int u) {
    q = q_ + s.first * qs_ + (size_t)kvh * v.group * RB;
    from_lse = lse_ + (size_t)s.first * v.n_head + kvh * v.group;
    qs = qs_;
    alike = ROWS % v.group == 0;
    offsets(v, b0 + u * ROWS);
  }
  __device__ __forceinline__ void offsets(const PagedView& v, int r0) {
    const int ta = quotient(r0, v.by_group);                        // offsets from there fit 32 bits
    auto from = [&](int r, int per_token, int per_head) INLINED {   // row b1 - 1 again behind the last
      const int row = min(r0 + r, b1 - 1), token = quotient(row, v.by_group);
      return (uint32_t)((token - ta) * per_token + (row - token * v.group) * per_head);
    };
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int r = (wave * NC + j) * RPC + lane / SEG;
      at[j] = from(r, (int)qs, RB) + ((lane % SEG) ^ swizzle(r)) * 16;
    }
    lse_at = from(lane, v.n_head * 4, 4);
  }
  __device__ __forceinline__ void issue(const PagedView& v, int u, int slot) {
    const int r0 = b0 + u * ROWS, ta = quotient(r0, v.by_group);
    if (!alike || r0 + 64 > b1) offsets(v, r0);
#pragma unroll
    for (int j = 0; j < NC; ++j) copy_to_lds(q + ta * qs, at[j], (u32x4_t*)(rows + slot * (ROWS * RB) + (wave * NC + j) * 1024));
    copy_words_to_lds((const char*)(from_lse + (size_t)ta * v.n_head), lse_at, lse + slot * 64);
  }
};

template <int DT, int D, bool SPLIT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void paged_weights_tile_kernel(
    PagedView v, const PagedKeys* __restrict__ blocks, const char* __restrict__ q, int64_t qs, const char* __restrict__ kc,
    const float* __restrict__ lse, float decay, float* __restrict__ w, int64_t ws) {
  constexpr bool F32 = DT == DT_F32;
  constexpr int RB = D * (F32 ? 4 : 2);
  constexpr int KG = F32 ? 2 : 1, KL = 32 / KG, KS = RB / (F32 ? 64 : 32);      // keys of a lane, lanes of a key group, operands of a row
  constexpr int ROWS = (F32 ? 32 : 64) / (SPLIT ? 2 : 1), X = ROWS / KL, RING = SPLIT ? 2 : 3, KEYS = SPLIT ? 32 : kWeighKeys;
  typedef QueryRing<RB, ROWS, SPLIT ? 1 : 4, RING> Ring;
  constexpr int NC = Ring::NC;
  __shared__ __attribute__((aligned(1024))) char rows_lds[SPLIT ? 4 : 1][RING][ROWS * RB];
  __shared__ __attribute__((aligned(1024))) float lse_lds[4][RING][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane / KL, n = lane % KL, kvh = blockIdx.x % v.n_kv;  // part of a row's operand, key of the group
  const PagedKeys block = uniform_load(blocks + blockIdx.x / v.n_kv);
  const PagedSeq s = uniform_load(v.seqs + block.seq);
  const int kb0 = block.key0 + blockIdx.y * KEYS;
  if (kb0 >= s.len) return;
  const int before = s.len - s.fresh, last16 = (s.len - 1) & ~15;
  const int k0 = SPLIT ? kb0 : kb0 + wave * 32;
  // rows that see some key of the block: [b0, b1); that see the lane's key: [lo, lo + number)
  const int b0 = first_token(s, kb0) * v.group, b1 = end_token(v, s, kb0, min(kb0 + KEYS, s.len)) * v.group;
  int lo[KG];
  uint32_t number[KG];
#pragma unroll
  for (int kg = 0; kg < KG; ++kg) {
    const int key = k0 + kg * KL + n;
    lo[kg] = first_token(s, key) * v.group;
    number[kg] = key < s.len ? (uint32_t)max(0, end_token(v, s, key, key + 1) * v.group - lo[kg]) : 0;
  }
  // ... of all of the wave's keys, of some of them
  const int oldest = max(k0, min(v.sinks, k0 + 31));                // the wave's key that drops out of the window first
  const int all0 = first_token(s, k0 + 31) * v.group, all1 = k0 + 32 > s.len ? 0 : end_token(v, s, oldest, oldest + 1) * v.group;
  const int any0 = first_token(s, k0) * v.group, any1 = k0 < s.len ? end_token(v, s, k0, min(k0 + 32, s.len)) * v.group : 0;
  const float c = v.scale * kLog2e;

  u32x4_t kf[KG][KS];
  {
    const int pl = min(k0, last16), ph = min(k0 + 16, last16);
    const uint32_t rl = cache_row(v, s, kvh, pl), rh = cache_row(v, s, kvh, ph);
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      const bool high = F32 ? kg == 1 : (n & 16) != 0;
      const char* kr = kc + (size_t)((high ? rh : rl) + min(n & 15, s.len - 1 - (high ? ph : pl))) * RB + h * 16;
#pragma unroll
      for (int i = 0; i < KS; ++i) kf[kg][i] = *(const u32x4_t*)(kr + i * (F32 ? 64 : 32));
    }
  }
  Ring ring;
  ring.rows = rows_lds[SPLIT ? wave : 0][0];
  ring.lse = lse_lds[wave][0];
  ring.b0 = b0;
  ring.b1 = b1;
  ring.wave = SPLIT ? 0 : wave;
  ring.lane = lane;
  ring.kvh = kvh;
  const uint32_t qaddr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&rows_lds[SPLIT ? wave : 0][0][0] +
                         (uint32_t)(n * RB + (h ^ Ring::swizzle(n)) * 16);
  const uint32_t laddr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)&lse_lds[wave][0][0];
  const int steps = b1 > b0 ? (b1 - b0 + ROWS - 1) / ROWS : 0;
  constexpr int BY = SPLIT ? 4 : 1;
  const int first = SPLIT ? wave : 0;
  float sum[KG][2];
#pragma unroll
  for (int kg = 0; kg < KG; ++kg) sum[kg][0] = sum[kg][1] = 0.f;
  if (first < steps) ring.start(v, s, q, qs, lse, first);
#pragma unroll
  for (int i = 0; i < RING - 1; ++i)
    if (first + i * BY < steps) ring.issue(v, first + i * BY, i);
  for (int u = first, slot = 0; u < steps; u += BY, slot = slot + 1 == RING ? 0 : slot + 1) {
    const int ahead = u + (RING - 1) * BY;
    if constexpr (SPLIT) {
      __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);                  // vmcnt(0): step u has landed
      asm volatile("" ::: "memory");
    } else {
      copies_barrier<(NC + 1) * (RING - 2)>(ahead - 1 >= steps);
    }
    if (ahead < steps) ring.issue(v, ahead, slot == 0 ? RING - 1 : slot - 1);
    const int r0 = b0 + u * ROWS, r1 = min(r0 + ROWS, b1);
    if (r1 <= any0 || r0 >= any1) continue;
    // lse of the step's rows in base 2, in place
    const uint32_t la = laddr + slot * 256;
    float mine;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(mine) : "v"(la + lane * 4) : "memory");
    asm volatile("ds_write_b32 %0, %1" ::"v"(la + lane * 4), "v"(mine * kLog2e) : "memory");
    uint32_t qa[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) qa[i] = (qaddr + slot * (ROWS * RB)) ^ (i * (F32 ? 64 : 32));
    const bool whole = r0 >= all0 && r0 + ROWS <= min(all1, b1);
    if constexpr (F32) {
      u32x4_t qf[X][KS], bits[X];             // lse of the lane's rows 16 x + 4 h + ..
      f32x4_t sacc[X][KG];
      read_pieces<0>(qa, qf[0]);
      if constexpr (X > 1) read_pieces<16 * RB>(qa, qf[X - 1]);
#pragma unroll
      for (int x = 0; x < X; ++x)
        asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(bits[x]) : "v"(la + x * 64 + h * 16) : "memory");
#pragma unroll
      for (int x = 0; x < X; ++x)
#pragma unroll
        for (int kg = 0; kg < KG; ++kg) sacc[x][kg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int x = 0; x < X; ++x)
#pragma unroll
            for (int kg = 0; kg < KG; ++kg)
              sacc[x][kg] = mfma_f32(__uint_as_float(qf[x][i][e]), __uint_as_float(kf[kg][i][e]), sacc[x][kg]);
#pragma unroll
      for (int x = 0; x < X; ++x)
#pragma unroll
        for (int kg = 0; kg < KG; ++kg)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = fmaf(sacc[x][kg][e], c, -__uint_as_float(bits[x][e]));
            const bool seen = (uint32_t)(r0 + x * 16 + 4 * h + e - lo[kg]) < number[kg];
            sum[kg][x & 1] += __builtin_amdgcn_exp2f(seen ? p : -INFINITY);
          }
    } else {
      f32x16_t sacc[X];
      uint32_t pa[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pa[i] = la + i * 32 + h * 16;
      u32x4_t bits[X][4];                     // lse of the lane's rows 8 i + 4 h + .. of each product
      auto product = [&](auto x_) INLINED {
        constexpr int x = decltype(x_)::value;
        u32x4_t qf[KS];
#pragma unroll
        for (int i = 0; i < 16; ++i) sacc[x][i] = 0.f;
        read_pieces<x * 32 * RB>(qa, qf);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sacc[x] = mfma32<DT>(qf[ks], kf[0][ks], sacc[x]);
      };
      product(std::integral_constant<int, 0>{});
      if constexpr (X > 1) product(std::integral_constant<int, X - 1>{});
      read_pieces<0>(pa, bits[0]);
      if constexpr (X > 1) read_pieces<128>(pa, bits[X - 1]);
      __builtin_amdgcn_s_setprio(1);
      auto add = [&](auto all) INLINED {
        const int r = r0 + 4 * h - lo[0];
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p = fmaf(sacc[x][i], c, -__uint_as_float(bits[x][i / 4][i % 4]));
            if constexpr (!decltype(all)::value) p = (uint32_t)(r + x * 32 + 8 * (i / 4) + i % 4) < number[0] ? p : -INFINITY;
            sum[0][x] += __builtin_amdgcn_exp2f(p);
          }
      };
      if (whole) add(std::true_type{});
      else add(std::false_type{});
      __builtin_amdgcn_s_setprio(0);
    }
  }
  // lane `key` of 32: the sum of key k0 + key
  float t = sum_partner<32>(sum[0][0] + sum[0][1]);
  if constexpr (F32) {
    const float t0 = sum_partner<16>(t), t1 = sum_partner<16>(sum_partner<32>(sum[KG - 1][0] + sum[KG - 1][1]));
    t = lane < 16 ? t0 : t1;
  }
  if constexpr (SPLIT) {
    __shared__ float sums[4][32];
    if (lane < 32) sums[wave][lane] = t;
    __syncthreads();
    if (wave > 0) return;
    t = lane < 32 ? (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]) : 0.f;
  }
  const int key = k0 + lane;
  if (lane < 32 && key < s.len) {
    float* to = w + ((int64_t)block.seq * v.n_kv + kvh) * ws + key;
    *to = new_weight(t, decay != 0.f && key < before ? *to : 0.f, decay, key >= before);
  }
}

// ---------------------------------------------------------------- eviction

// Order of a weight: larger is heavier, NaN the lightest, both zeros alike.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// A block per (key head, sequence).  The weight of the last row kept is found digit by digit from the top (four digits of 8 bits, counted
// in LDS); rows of exactly that weight are taken from the front.  Then the positions are gone through in order, four per thread, and numbered.  The
// weights' keys stay in LDS (the first kKeysHeld of them; of a longer sequence the rest is read again).  32 sequences of up to 4096 rows, 8 key heads:
// 9.8 us, a chain of dependent steps.
constexpr int kKeysHeld = 18432;           // 72 KB: two blocks per compute unit
// Sums over the lanes up to and including one's own, of the wave; lanes without a source add zero.
template <int CTRL, int ROWS> __device__ __forceinline__ int plus_dpp(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int scan16(int x) {               // within 16 lanes: row_shr 1, 2, 4, 8
  return plus_dpp<0x118, 0xf>(plus_dpp<0x114, 0xf>(plus_dpp<0x112, 0xf>(plus_dpp<0x111, 0xf>(x))));
}
__device__ __forceinline__ int scan64(int x) {               // lane 15 of rows 0 and 2 to rows 1 and 3, lane 31 to rows 2 and 3
  return plus_dpp<0x143, 0xc>(plus_dpp<0x142, 0xa>(scan16(x)));
}
__global__ __launch_bounds__(1024) void paged_select_kernel(PagedView v, const float* w, int64_t ws, int budget, int first,
                                                            int recent, float* wo, int64_t os, int* __restrict__ kept) {
  __shared__ uint32_t held[kKeysHeld];
  __shared__ int count[256];
  __shared__ int found[3];                 // digit, rows still wanted of it, whether those are all
  __shared__ int waves[2][16][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t at = (size_t)blockIdx.y * v.n_kv + blockIdx.x;
  const int len = uniform_load(&v.seqs[blockIdx.y].len);
  const float* mine = w + at * ws;
  float* to = wo ? wo + at * os : nullptr;
  int* keep = kept + at * budget;
  if (len <= budget) {
    for (int p = tid; p < budget; p += 1024) {
      keep[p] = p < len ? p : -1;
      if (to && p < len && (wo != w)) to[p] = mine[p];
    }
    return;
  }
  if (tid < 256) count[tid] = 0;
  for (int p0 = 0; p0 < min(len, kKeysHeld); p0 += 4096) {      // four loads on their way at a time
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = mine[min(p0 + j * 1024 + tid, len - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p0 + j * 1024 + tid < min(len, kKeysHeld)) held[p0 + j * 1024 + tid] = weight_key(x[j]);
  }
  auto key_of = [&](int p) INLINED { return p < kKeysHeld ? held[p] : weight_key(mine[p]); };
  const int sure = first + recent;         // of the others, `wanted` are kept
  int wanted = budget - sure;
  uint32_t prefix = 0;
  bool whole = false;
  for (int shift = 24; shift >= 0 && wanted > 0 && !whole; shift -= 8) {
    __syncthreads();
    for (int p = first + tid; p < len - recent; p += 1024) {
      const uint32_t k = key_of(p);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&count[k >> shift & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {                       // lane l: digits 255 - 4l and the three below
      int c[4], sum = 0;
      for (int i = 0; i < 4; ++i) {
        sum += c[i] = count[255 - 4 * lane - i];
        count[255 - 4 * lane - i] = 0;
      }
      const int upto = scan64(sum);
      if (lane == __builtin_ctzll(__ballot(upto >= wanted))) {      // the rows under way are more than `wanted`
        int left = wanted - (upto - sum), i = 0;
        while (i < 3 && c[i] < left) left -= c[i++];
        found[0] = 255 - 4 * lane - i;
        found[1] = left;
        found[2] = left == c[i];            // every row that begins with these digits: the others need not be known
      }
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    wanted = found[1];
    whole = found[2];
  }
  // heavier than prefix (or as heavy, where all of those are kept): kept; equal: the first `wanted`
  int ranks = 0, ties = 0;                 // kept, and equal ones met, so far
  for (int p0 = 0, turn = 0; p0 < len; p0 += 4096, turn ^= 1) {
    const int first_p = p0 + tid * 4;
    float x[4];
    uint32_t above = 0, tie = 0;           // bits: of the thread's four positions
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = first_p + j;
      x[j] = to && p < len ? mine[p] : 0.f;
      const uint32_t k = p < len ? key_of(p) : 0u;
      const bool certain = p < len && (p < first || p >= len - recent), middle = p < len && !certain && budget > sure;
      above |= (uint32_t)(certain || (middle && (k > prefix || (whole && k == prefix)))) << j;
      tie |= (uint32_t)(middle && !whole && k == prefix) << j;
    }
    const int te = __popc(tie), ta = __popc(above), se = scan64(te), sa = scan64(ta);
    if (lane == 63) {
      waves[turn][wave][0] = se;
      waves[turn][wave][1] = sa;
    }
    __syncthreads();                       // (the other turn's counts are read before the next barrier)
    // in front of the wave: equal ones, of which the first `wanted` are kept, and kept ones.  Lane i sums up for wave i
    const int e = lane < 16 ? waves[turn][lane][0] : 0, e_upto = scan16(e);
    const int more = lane < 16 ? waves[turn][lane][1] + max(0, min(e, wanted - ties - (e_upto - e))) : 0, more_upto = scan16(more);
    const int of_wave = ties + __builtin_amdgcn_readlane(e_upto - e, wave);
    int t = of_wave + se - te;
    int r = ranks + __builtin_amdgcn_readlane(more_upto - more, wave) + (sa - ta) + min(t, wanted) - min(of_wave, wanted);
    ties += __builtin_amdgcn_readlane(e_upto, 15);
    ranks += __builtin_amdgcn_readlane(more_upto, 15);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool equal = tie >> j & 1;
      if ((above >> j & 1) || (equal && t < wanted)) {
        keep[r] = first_p + j;
        if (to) to[r] = x[j];              // at or in front of its own: behind the barrier nobody reads that place any more
        ++r;
      }
      t += equal;
    }
  }
}

// The kept rows to the front: block = (PIECES x 16 bytes of a row, key head, sequence x K|V), 256 threads, PIECES per row, kMove rows of each thread
// at a time.
// A row moves to a place at or in front of its own, and a place is overwritten only once every row up to it has been read: a
// barrier between the reads (waited for) and the writes of a batch is enough, because the batch behind reads from places behind.  Where the rows of
// the next batch lie and go is looked up, a row per thread, while a batch is read.  28 sequences to 1024 rows of 8 x 256 bytes, K and V: 45 to 52 us.
// 128 bytes of a row where there are blocks enough, otherwise 32: four times the blocks, and a quarter of the batches one after the other.
constexpr int kMove = 8;
template <int PIECES>
__global__ __launch_bounds__(256) void paged_move_kernel(PagedView v, char* kc, char* vc, int budget, int first,
                                                         const int* __restrict__ kept, int row_bytes) {
  constexpr int PER = 256 / PIECES, STEP = PER * kMove, EACH = STEP / 256;      // rows of a pass, of a batch, of a batch per thread
  __shared__ uint2 rows[2][STEP];            // of a batch, in turns: (from, to)
  const PagedSeq s = uniform_load(v.seqs + (blockIdx.z >> 1));
  if (s.len <= budget) return;
  const int kvh = blockIdx.y, tid = threadIdx.x;
  char* cache = (blockIdx.z & 1 ? vc : kc) + blockIdx.x * (PIECES * 16) + tid % PIECES * 16;
  const int* keep = kept + ((size_t)(blockIdx.z >> 1) * v.n_kv + kvh) * budget;
  struct Lookup {
    int pos[EACH], from[EACH], to[EACH];
  };
  auto positions = [&](Lookup& a, int r0) INLINED {
#pragma unroll
    for (int i = 0; i < EACH; ++i) a.pos[i] = keep[min(r0 + i * 256 + tid, budget - 1)];
  };
  auto pages = [&](Lookup& a, int r0) INLINED {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      a.from[i] = v.pages[s.pages + quotient(a.pos[i], v.by_page)];
      a.to[i] = v.pages[s.pages + quotient(min(r0 + i * 256 + tid, budget - 1), v.by_page)];
    }
  };
  auto row = [&](int page, int pos) INLINED { return ((uint32_t)page * v.n_kv + kvh) * v.page_size + (pos - quotient(pos, v.by_page) * v.page_size); };
  auto put = [&](int turn, const Lookup& a, int r0) INLINED {
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      rows[turn][i * 256 + tid] = make_uint2(row(a.from[i], a.pos[i]), row(a.to[i], min(r0 + i * 256 + tid, budget - 1)));
  };
  Lookup ahead;
  positions(ahead, first);
  pages(ahead, first);
  put(0, ahead, first);
  positions(ahead, first + STEP);
  __syncthreads();
  for (int r0 = first, turn = 0; r0 < budget; r0 += STEP, turn ^= 1) {
    pages(ahead, r0 + STEP);
    u32x4_t x[kMove];
    uint32_t to[kMove];
#pragma unroll
    for (int j = 0; j < kMove; ++j) {
      const uint2 ft = rows[turn][j * PER + tid / PIECES];
      to[j] = ft.y;
      x[j] = *(const u32x4_t*)(cache + (size_t)ft.x * row_bytes);
    }
    put(turn ^ 1, ahead, r0 + STEP);
    positions(ahead, r0 + 2 * STEP);
#pragma unroll
    for (int j = 0; j < kMove; ++j) asm volatile("" : "+v"(x[j]));      // has been read
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMove; ++j)
      if (r0 + j * PER + tid / PIECES < budget) *(u32x4_t*)(cache + (size_t)to[j] * row_bytes) = x[j];
  }
}

// f(std::integral_constant dtype, head_dim)
template <class F> void with_types(int dtype, int d, F f) {
  auto wide = [&](auto dt) {
    if (d == 128) f(dt, std::integral_constant<int, 128>{});
    else f(dt, std::integral_constant<int, 64>{});
  };
  if (dtype == DT_F32) wide(std::integral_constant<int, DT_F32>{});
  else if (dtype == DT_F16) wide(std::integral_constant<int, DT_F16>{});
  else wide(std::integral_constant<int, DT_BF16>{});
}
int element_bytes(int dtype) { return dtype == DT_F32 ? 4 : 2; }

}  // namespace

hipError_t paged_append(int dtype, const PagedView& v, const void* k, int64_t ks, const void* vv, int64_t vs, void* kc, void* vc, hipStream_t st) {
  const int eb = element_bytes(dtype), pieces = v.d * eb / 16;
  const int64_t blocks = ((int64_t)v.tokens * v.n_kv * pieces + 255) / 256;
  paged_append_kernel<<<dim3((unsigned)blocks, 2), 256, 0, st>>>(v, (const char*)k, ks * eb, (const char*)vv, vs * eb, (char*)kc, (char*)vc, pieces);
  return hipGetLastError();
}

hipError_t paged_attention(int dtype, const PagedView& v, const PagedItem* rows, int n_rows, const PagedItem* tiles, int n_tiles,
                           const PagedMerge* merges, int n_merges, int most_parts, int most_rows,
                           const void* q, int64_t qs, const void* kc, const void* vc, void* out, float* lse, hipStream_t st) {
  with_types(dtype, v.d, [&](auto dt, auto d) {
    constexpr int DT = decltype(dt)::value, D = decltype(d)::value;
    if constexpr (DT != DT_F32)
      if (n_tiles) paged_tile_kernel<DT, D><<<n_tiles * v.n_kv, 256, 0, st>>>(v, tiles, (const char*)q, qs * 2, (const char*)kc,
                                                                              (const char*)vc, out, lse);
    if (n_rows) paged_rows_kernel<DT, D><<<n_rows * v.n_kv, 256, 0, st>>>(v, rows, (const char*)q, qs * element_bytes(DT), (const char*)kc,
                                                                          (const char*)vc, out, lse);
    if (n_merges) {
      if (most_parts > 8) paged_merge_kernel<DT, D, 4><<<dim3(n_merges * v.n_kv, most_rows), 256, 0, st>>>(v, merges, out, lse);
      else paged_merge_kernel<DT, D, 1><<<dim3(n_merges * v.n_kv, (most_rows + 3) / 4), 256, 0, st>>>(v, merges, out, lse);
    }
  });
  return hipGetLastError();
}

hipError_t paged_weights(int dtype, const PagedView& v, const void* q, int64_t qs, const void* kc, const float* lse, float decay, float* w,
                         int64_t ws, bool few, bool few_blocks, const PagedKeys* many, int n_many, bool split, hipStream_t st) {
  with_types(dtype, v.d, [&](auto dt, auto d) {
    constexpr int DT = decltype(dt)::value, D = decltype(d)::value;
    const int64_t qb = qs * element_bytes(DT);
    // Two steps of a wave per block while the blocks are few, four then: 1 sequence of 8192 rows, 8 key heads 8.3 -> 6.6 us, 8 of up to 2000 8.9 -> 8.0;
    // 64 of up to 8192 117 -> 112, 200 of up to 512 24.1 -> 21.7
    const int keys = few_blocks ? 256 : 512;
    if (few) paged_weights_rows_kernel<DT, D><<<dim3((v.longest + keys - 1) / keys, v.n_kv, v.n_seq), 256, 0, st>>>(
        v, (const char*)q, qb, (const char*)kc, lse, decay, w, ws, keys);
    if (n_many > 0) {
      if (split)
        paged_weights_tile_kernel<DT, D, true><<<dim3(n_many * v.n_kv, kWeighKeys / 32), 256, 0, st>>>(
            v, many, (const char*)q, qb, (const char*)kc, lse, decay, w, ws);
      else
        paged_weights_tile_kernel<DT, D, false><<<n_many * v.n_kv, 256, 0, st>>>(v, many, (const char*)q, qb, (const char*)kc, lse, decay, w, ws);
    }
  });
  return hipGetLastError();
}

hipError_t paged_evict(int dtype, const PagedView& v, void* kc, void* vc, const float* w, int64_t ws, int budget, int first, int recent,
                       float* wo, int64_t os, int* kept, hipStream_t st) {
  paged_select_kernel<<<dim3(v.n_kv, v.n_seq), 1024, 0, st>>>(v, w, ws, budget, first, recent, wo, os, kept);
  const int row_bytes = v.d * element_bytes(dtype);
  if (v.longest > budget) {
    const int heads = 2 * v.n_seq * v.n_kv;
    if (heads * (row_bytes / 128) >= 256)
      paged_move_kernel<8><<<dim3(row_bytes / 128, v.n_kv, 2 * v.n_seq), 256, 0, st>>>(v, (char*)kc, (char*)vc, budget, first, kept, row_bytes);
    else
      paged_move_kernel<2><<<dim3(row_bytes / 32, v.n_kv, 2 * v.n_seq), 256, 0, st>>>(v, (char*)kc, (char*)vc, budget, first, kept, row_bytes);
  }
  return hipGetLastError();
}

}  // namespace flk
