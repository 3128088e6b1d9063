// Rotary positions, and the append of a block's keys and values to the paged cache.
//
// Both are streams: every element is read once and written once, and a rotated pair costs a few
// multiply-adds, so memory bounds them (or, for a few rows, the launch and its chain of loads).  A
// thread keeps one unit of a head -- the same 16-byte piece, or pair of pieces, in every head -- of one row:
// it forms that unit's cosines and sines once, in registers, and then walks the heads with four
// loads in flight.  (A wave for every head, which formed them anew: 55 us where this takes 27.7.)
// Times are the kernel's, in a captured graph.
#include "lsv_attn.h"
#include "lsv_ops.h"

namespace lsv {

constexpr int kThreads = 256;
constexpr int kPage = LSV_KV_PAGE;

// amplitude * (cos, sin) of a pair at a position: the product in fp64, reduced to [-1, 1] half turns.  The reduced angle is
// rounded to fp32, which moves a rotated element by 2^-23.3 of the pair at most, less than its sine's and its own
// roundings to fp32 together (2^-22); sines in fp64 would be stored in no more bits.
LSV_DEV float2 rope_turn(float amplitude, double half_turns, int pos) {
  const double t = (double)pos * half_turns;
  float sn, cs;
  sincospif((float)(t - 2.0 * rint(0.5 * t)), &sn, &cs);
  return make_float2(amplitude * cs, amplitude * sn);
}

template <typename T, int N> struct Piece {
  T e[N];
};
template <typename T, int N> LSV_DEV Piece<T, N> load_piece(const T* p) {
  if constexpr (N == 1) return Piece<T, 1>{GL(p)[0]};
  else return __builtin_bit_cast(Piece<T, N>, *(const GLOBAL u32x4_t*)(const GLOBAL T*)GL(p));
}
// Non-temporal: what is written is read by another kernel, through the memory-side cache at best (8191 rows
// of 40 heads: 37.9 us with default stores, 27.7 with these, 30.7 with non-temporal loads instead, 33.7 with
// both; a layer's append and attention together take the same time either way).
template <typename T, int N> LSV_DEV void store_piece(T* p, const Piece<T, N>& v) {
  if constexpr (N == 1) GL(p)[0] = v.e[0];
  else __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), (GLOBAL u32x4_t*)(GLOBAL T*)GL(p));
}

// How a rotation is spread over a workgroup's threads.  VEC: a unit is a piece of 16 bytes (HALF: one in
// each half of the pairs); else one pair.  Behind the rotated units come those of the tail, copied.
struct Units {
  int turned, per_head;  // units of a head
};
__host__ __device__ inline Units units_of(int layout, int rot, int hd, int n, bool copy) {
  Units u;
  u.turned = layout == LSV_ROPE_HALF || n == 1 ? rot / 2 / n : rot / n;
  u.per_head = u.turned + (copy ? (hd - rot) / n : 0);
  return u;
}

// Rotate `nrow` rows of `heads` heads: from(r, h) and to(r, h) are head h of row r, pos(r, p) sets the row's
// position, false: the row stays as it is.  Threads take (unit, row, head) with the unit fastest.  A thread owns
// both elements of its pairs, so that rotating in place is safe; the unrotated tail goes over only where `copy` says so.
template <typename T, bool VEC, bool HALF, typename From, typename To, typename Pos>
LSV_DEV void rotate_rows(const RopeArgs& rope, int nrow, int heads, int hd, bool copy, From from, To to, Pos pos) {
  constexpr int N = VEC ? 16 / (int)sizeof(T) : 1;   // elements of a piece
  constexpr int TWO = HALF || !VEC ? 2 : 1;          // pieces of a unit
  constexpr int PAIRS = N * TWO / 2, BATCH = 4;
  const Units un = units_of(HALF ? LSV_ROPE_HALF : LSV_ROPE_INTERLEAVED, rope.rot, hd, N, copy);
  if (un.per_head == 0) return;
  const int rows = min(nrow, kThreads / un.per_head), lanes = kThreads / (un.per_head * rows);
  const int u = threadIdx.x % un.per_head, rest = threadIdx.x / un.per_head, r0 = rest % rows, h0 = rest / rows;
  if (h0 >= lanes) return;
  const bool turns = u < un.turned;
  // elements of the unit's pieces within a head
  const int ea = turns ? (HALF || VEC ? u * N : 2 * u) : rope.rot + (u - un.turned) * N;
  const int eb = HALF ? ea + rope.rot / 2 : ea + 1;
  double f[PAIRS];
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) f[k] = turns ? rope.half_turns[(HALF || !VEC ? u * N : u * N / 2) + k] : 0.0;
  for (int r = r0; r < nrow; r += rows) {
    int p;
    if (!pos(r, p)) continue;
    float2 c[PAIRS];
    bool formed = false;
    for (int h = h0; h < heads; h += lanes * BATCH) {
      Piece<T, N> a[BATCH], b[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int hk = h + k * lanes;
        if (hk < heads) {
          const T* x = from(r, hk);
          a[k] = load_piece<T, N>(x + ea);
          if (TWO == 2 && turns) b[k] = load_piece<T, N>(x + eb);
        }
      }
      if (!formed && turns) {  // behind the first loads
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) c[k] = rope_turn(rope.amplitude, f[k], p);
        formed = true;
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int hk = h + k * lanes;
        if (hk >= heads) break;
        T* y = to(r, hk);
        if (turns) {
#pragma unroll
          for (int e = 0; e < PAIRS; ++e) {
            T& first = TWO == 2 ? a[k].e[e] : a[k].e[2 * e % N];
            T& second = TWO == 2 ? b[k].e[e] : a[k].e[(2 * e + 1) % N];
            const float v = to_f32<T>(first), w = to_f32<T>(second);
            first = from_f32<T>(v * c[e].x - w * c[e].y);
            second = from_f32<T>(w * c[e].x + v * c[e].y);
          }
          if (TWO == 2) store_piece<T, N>(y + eb, b[k]);
        }
        store_piece<T, N>(y + ea, a[k]);
      }
    }
  }
}

// Whether units of 16-byte pieces can be taken: pieces that lie in one half of the pairs.
static bool pieces_fit(const RopeArgs& rope, int hd, size_t es) {
  const int n = (int)(16 / es);
  return hd % n == 0 && rope.rot % n == 0 && (rope.layout != LSV_ROPE_HALF || (rope.rot / 2) % n == 0);
}
static bool aligned16(const void* p, int64_t stride, size_t es) {
  return ((uintptr_t)p & 15) == 0 && (stride * (int64_t)es) % 16 == 0;
}

// ------------------------------------------------------------------ rotation of a row array
// A workgroup takes `group` rows and `lot` heads.  8191 rows of 40 heads of 128: 168 MB in 27.7 us, 6.1 TB/s (a copy of
// 1 GiB moves 5.1); 32 rows: 4.0 us by positions, the launch, 4.9 as 32 sequences by their lengths.
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs rope, RowArgs rows, int group, int lot, const T* x,
                                                        int64_t xs, T* y, int64_t ys, int heads, int hd, bool copy) {
  // per sequence: its first row; the row behind it and those before it; its position minus its row
  __shared__ int begin[LSV_MAX_BATCH], end[LSV_MAX_BATCH], base[LSV_MAX_BATCH];
  const int first = rows.row_offsets ? GL(rows.row_offsets)[0] : 0;
  const int M = rows.row_offsets ? GL(rows.row_offsets)[rows.batch] : rows.max_rows;
  if (!rows.positions) {  // its loads go out with those of first and M
    const SeqRows s = seq_rows(rows);
    const int behind = wave_scan_max(s.rows > 0 ? s.r0 + s.rows : 0), t = threadIdx.x;
    if (t < rows.batch) {
      begin[t] = s.r0;
      end[t] = behind;
      base[t] = s.C - s.r0;
    }
    __syncthreads();
  }
  if (first < 0 || first > M || M > rows.max_rows) return;
  const int m0 = first + blockIdx.x * group, h0 = blockIdx.y * lot;
  if (m0 >= M) return;
  auto pos = [&](int r, int& p) {
    const int m = m0 + r;
    if (rows.positions) {
      p = GL(rows.positions)[m];
      return true;
    }
    int b = 0;  // the ends rise: as many sequences lie before the row as end at or before it
    for (int k = 0; k + 1 < rows.batch; ++k) b += end[k] <= m ? 1 : 0;
    p = base[b] + m;
    return m >= begin[b] && m < end[b];  // else a refused sequence's row
  };
  const T* px = x + m0 * xs + (int64_t)h0 * hd;
  T* py = y + m0 * ys + (int64_t)h0 * hd;
  rotate_rows<T, VEC, HALF>(rope, min(group, M - m0), min(lot, heads - h0), hd, copy,
                            [&](int r, int h) { return px + r * xs + (int64_t)h * hd; },
                            [&](int r, int h) { return py + r * ys + (int64_t)h * hd; }, pos);
}

// One row a workgroup and one unit a thread until the workgroups fill the chip; then as many rows as the
// threads hold at once, and up to eight heads a thread, which share its angles.
template <typename T, bool VEC, bool HALF>
static void launch_rope_form(const RopeArgs& rope, int heads, int hd, const RowArgs& rows, const T* x, int64_t xs, T* y,
                             int64_t ys, hipStream_t st) {
  const bool copy = x != y;
  const int units = units_of(rope.layout, rope.rot, hd, VEC ? 16 / (int)sizeof(T) : 1, copy).per_head;
  const int most = kThreads / units, want = rows.max_rows / 256;
  const int group = want < 1 ? 1 : want > most ? most : want;
  const int lanes = kThreads / (units * group), lot = lanes * (want < 1 ? 1 : want > 8 ? 8 : want);
  hipLaunchKernelGGL((rope_kernel<T, VEC, HALF>), dim3((rows.max_rows + group - 1) / group, (heads + lot - 1) / lot),
                     dim3(kThreads), 0, st, rope, rows, group, lot, x, xs, y, ys, heads, hd, copy);
}

template <typename T>
static int launch_rope_t(const RopeArgs& rope, int heads, int hd, const RowArgs& rows, const void* vx, int64_t xs,
                         void* vy, int64_t ys, hipStream_t st) {
  const T* x = (const T*)vx;
  T* y = (T*)vy;
  const bool vec = pieces_fit(rope, hd, sizeof(T)) && aligned16(x, xs, sizeof(T)) && aligned16(y, ys, sizeof(T));
  if (rope.layout == LSV_ROPE_HALF) {
    if (vec) launch_rope_form<T, true, true>(rope, heads, hd, rows, x, xs, y, ys, st);
    else launch_rope_form<T, false, true>(rope, heads, hd, rows, x, xs, y, ys, st);
  } else {
    if (vec) launch_rope_form<T, true, false>(rope, heads, hd, rows, x, xs, y, ys, st);
    else launch_rope_form<T, false, false>(rope, heads, hd, rows, x, xs, y, ys, st);
  }
  return hipGetLastError() == hipSuccess ? LSV_OK : LSV_ERR_HIP;
}

int launch_rope(const RopeArgs& rope, int dtype, int heads, int hd, const RowArgs& rows, const void* x, int64_t xs,
                void* y, int64_t ys, hipStream_t st) {
  return dtype == LSV_DTYPE_BF16 ? launch_rope_t<bf16_t>(rope, heads, hd, rows, x, xs, y, ys, st)
                                 : launch_rope_t<float>(rope, heads, hd, rows, x, xs, y, ys, st);
}

// ------------------------------------------------------------------ append
// A workgroup takes the rows of one sequence that fall into one page (blockIdx.x counts these page
// runs over the sequences) and one kv head with its query heads: up to 64 rows.  4095 rows of 64 + 8 + 8 heads: 168 MB in
// 32.0 us, 5.2 TB/s; 32 sequences of one token: 6.1 us, bound by its chain of loads.  V goes through LDS:
// rows come in along the head, the page wants them along the positions, eight permuted columns to
// 16 or 32 bytes.  Its loads are the first, its stores the last.
template <typename T, int HD, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads) append_kernel(RopeArgs rope, AppendArgs a) {
  constexpr int N = VEC ? 16 / (int)sizeof(T) : 1, P = HD / N;  // elements of a piece, pieces of a V row
  constexpr int V = VEC ? kPage * P / kThreads : 1;             // pieces of V a thread
  __shared__ __align__(16) T Vl[kPage * HD];
  // V of key j, element d, in LDS: rows turned by eight banks per key group, so that a wave's reads of
  // its eight groups hit separate banks and 16-byte pieces stay whole
  auto v_at = [&](int j, int d) {
    const int group = ((j >> 2) & 3) | ((j >> 5) << 2);
    return j * HD + ((d + group * (32 / (int)sizeof(T))) & (HD - 1));
  };

  const int kvh = blockIdx.y;
  const SeqRows s = seq_rows(a.rows);
  if (a.status && blockIdx.x == 0 && kvh == 0 && (int)threadIdx.x < a.rows.batch) a.status[threadIdx.x] = s.status;
  const int runs = s.rows > 0 ? (s.C + s.rows - 1) / kPage - s.C / kPage + 1 : 0;
  const int sum = wave_scan_sum(runs);
  const int unit = blockIdx.x;
  const unsigned long long past = __ballot(sum > unit);
  if (!past) return;
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
  const int C = __builtin_amdgcn_readlane(s.C, b), rows = __builtin_amdgcn_readlane(s.rows, b);
  const int p = C / kPage + unit - __builtin_amdgcn_readlane(sum - runs, b);  // the page's index in the sequence
  const int first = max(C, p * kPage), n = min(C + rows, (p + 1) * kPage) - first;
  const int m0 = __builtin_amdgcn_readlane(s.r0, b) + first - C, j0 = first - p * kPage;
  const int page = GL(a.kv.pages)[(size_t)b * a.kv.max_pages + p];

  const T* v = (const T*)a.v + m0 * a.vs + (int64_t)kvh * HD;
  Piece<T, N> held[V];
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int i = k * kThreads + threadIdx.x, r = i / P, e = i % P * N;
      if (r < n) held[k] = load_piece<T, N>(v + r * a.vs + e);
    }
  }
  const bool there = page >= 0 && page < a.kv.n_pages;
  const size_t block = ((size_t)(there ? page : 0) * a.nkv + kvh) * kPage * HD;
  // the head's queries, then its key as one head more (left out where it has no page)
  const int group = a.nq / a.nkv;
  const T* q = (const T*)a.q + m0 * a.qs + (int64_t)kvh * group * HD;
  const T* k = (const T*)a.k + m0 * a.ks + (int64_t)kvh * HD;
  T* q_out = (T*)a.q_out + m0 * a.qos + (int64_t)kvh * group * HD;
  T* k_out = (T*)a.k_pool + block + (size_t)j0 * HD;
  rotate_rows<T, VEC, HALF>(rope, n, group + (there ? 1 : 0), HD, true,
                            [&](int r, int h) { return h < group ? q + r * a.qs + (int64_t)h * HD : k + r * a.ks; },
                            [&](int r, int h) { return h < group ? q_out + r * a.qos + (int64_t)h * HD : k_out + r * HD; },
                            [&](int r, int& p) {
                              p = a.rows.positions ? GL(a.rows.positions)[m0 + r] : first + r;
                              return true;
                            });
  if (!there) return;
  if constexpr (VEC) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int i = k * kThreads + threadIdx.x, r = i / P, e = i % P * N;
      if (r < n) *(Piece<T, N>*)&Vl[v_at(j0 + r, e)] = held[k];
    }
  } else {
    for (int i = threadIdx.x; i < n * HD; i += kThreads) Vl[v_at(j0 + i / HD, i % HD)] = GL(v)[i / HD * a.vs + i % HD];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < HD * 8; i += kThreads) {
    const int d = i >> 3, cg = i & 7;
    const int k0 = (cg >> 2) * 32 + (cg & 3) * 4;  // columns 8 cg + e hold keys k0 + e, k0 + 16 + e, e < 4
    T* dst = (T*)a.v_pool + block + (size_t)d * kPage + 8 * cg;
    if (k0 >= j0 && k0 + 19 < j0 + n) {
      T e[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e[k] = Vl[v_at(k0 + k, d)];
        e[4 + k] = Vl[v_at(k0 + 16 + k, d)];
      }
      constexpr int W = 16 / (int)sizeof(T);
#pragma unroll
      for (int k = 0; k < 8; k += W) {
        Piece<T, W> x;
#pragma unroll
        for (int l = 0; l < W; ++l) x.e[l] = e[k + l];
        store_piece<T, W>(dst + k, x);
      }
    } else {  // the run begins or ends inside the group: only its own columns
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int key = k0 + (k & 3) + (k >> 2) * 16;
        if (key >= j0 && key < j0 + n) dst[k] = Vl[v_at(key, d)];
      }
    }
  }
}

template <typename T, int HD> static int launch_append_t(const RopeArgs& rope, const AppendArgs& a, hipStream_t st) {
  // page runs of B' sequences with M rows: at most one a row, and (rows + 62) / 64 + 1 for each sequence
  const int M = a.rows.max_rows, B = a.rows.batch < M ? a.rows.batch : M;
  const long long most = ((long long)M + 62ll * B) / kPage + B;
  const dim3 grid((unsigned)(most < M ? most : M), (unsigned)a.nkv), block(kThreads);
  const bool vec = pieces_fit(rope, HD, sizeof(T)) && aligned16(a.k, a.ks, sizeof(T)) && aligned16(a.v, a.vs, sizeof(T)) &&
                   (!a.nq || (aligned16(a.q, a.qs, sizeof(T)) && aligned16(a.q_out, a.qos, sizeof(T))));
  if (rope.layout == LSV_ROPE_HALF) {
    if (vec) hipLaunchKernelGGL((append_kernel<T, HD, true, true>), grid, block, 0, st, rope, a);
    else hipLaunchKernelGGL((append_kernel<T, HD, false, true>), grid, block, 0, st, rope, a);
  } else {
    if (vec) hipLaunchKernelGGL((append_kernel<T, HD, true, false>), grid, block, 0, st, rope, a);
    else hipLaunchKernelGGL((append_kernel<T, HD, false, false>), grid, block, 0, st, rope, a);
  }
  return hipGetLastError() == hipSuccess ? LSV_OK : LSV_ERR_HIP;
}

int launch_append(const RopeArgs& rope, int dtype, const AppendArgs& a, hipStream_t st) {
  if (dtype == LSV_DTYPE_BF16) return a.hd == 128 ? launch_append_t<bf16_t, 128>(rope, a, st) : launch_append_t<bf16_t, 64>(rope, a, st);
  return a.hd == 128 ? launch_append_t<float, 128>(rope, a, st) : launch_append_t<float, 64>(rope, a, st);
}

}  // namespace lsv
