// Softmax attention over the keys and values of a cache in pages: whole sequences behind prefixes that
// they may share, and the pages chosen for every token and key head.
//
// Rows, tiles and arithmetic are those of the packed attention (tdq_attention.hip): the query heads of a
// key head are rows of one tile, a wavefront has 32 of them.  Here the keys of a tile come in granules of
// 16, the smallest page, each from where the table says.
#include "tdq_attend.hpp"
#include "tdq_pages.hpp"

namespace tdq {

constexpr int kGranule = 16, kGranuleBits = 4;
constexpr int kNowhere = 1 << 30;      // key of a granule that no row sees (a page that is not there)

// Where a granule is: its page (negative: not there), and the key that its first row is.
struct Granule {
  int page, key;
};

// One of the cache's two tensors.
struct Pages {
  const void* data;
  long long page, token, head;
};

// Copies of a granule's rows to LDS, 64 lanes with 16 bytes each a copy; rows of LDS have DP elements,
// their pieces at PLACE.
template <typename T, int DP, int PLACE(int)>
struct GranuleCopy {
  static constexpr int PIECES = DP / 8, ROWS = 64 / PIECES, N = kGranule / ROWS;
  u32 off[N];                          // bytes from the granule's first row (whole granules)
  u32 mine;                            // bit i: whether the head has what this lane copies in copy i

  __device__ __forceinline__ GranuleCopy(long long token, int D, int lane) {
    mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = i * ROWS + lane / PIECES, piece = (lane % PIECES) ^ PLACE(row);
      off[i] = (u32)(row * token * 2) + 16 * piece;
      mine |= (u32)(8 * piece < D) << i;
    }
  }
  // All rows; where D < DP the pieces past it keep what LDS holds.  `once`: nobody else reads them.
  __device__ __forceinline__ void whole(const T* first, u32 lds, bool full, bool once) const {
    if (full && once) {
#pragma unroll
      for (int i = 0; i < N; ++i) stream_to_lds(first, off[i], lds + 1024 * i);
    } else if (full) {
#pragma unroll
      for (int i = 0; i < N; ++i) copy_to_lds(first, off[i], lds + 1024 * i);
    } else if (once) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (mine >> i & 1) stream_to_lds(first, off[i], lds + 1024 * i);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (mine >> i & 1) copy_to_lds(first, off[i], lds + 1024 * i);
    }
  }
  // The first `left` rows, zeros behind them and past D.
  __device__ __forceinline__ void some(const T* first, long long token, int left, u32 lds) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = i * ROWS + lane / PIECES, piece = (lane % PIECES) ^ PLACE(row);
      const T* p = first + row * token + 8 * piece;
      copy_to_lds(row < left && (mine >> i & 1) ? (const void*)p : (const void*)kZeros, lds + 1024 * i);
    }
  }
};

// The granules of a sequence, in order.  (Any i, as long as there is a key.)
struct Line {
  const int* table;                    // the sequence's pages
  int shift, n_pages, keys;
  bool sure;                           // all pages of interest are there
  __device__ __forceinline__ Granule operator()(int i) const {
    const int last = (keys - 1) >> kGranuleBits, at = i < last ? i : last;
    const int page = table[at >> (shift - kGranuleBits)];
    const bool there = i <= last && page >= 0 && page < n_pages;
    return {there ? page : -1, there ? i << kGranuleBits : kNowhere};
  }
  // Looks at the pages of granules lo to hi.
  __device__ __forceinline__ void look_over(int lo, int hi) {
    sure = true;
    if (keys <= 0) return;
    const int bits = shift - kGranuleBits, last = (keys - 1) >> shift;
    int end = (hi - 1) >> bits;
    end = end < last ? end : last;
    for (int b = (lo >> bits) + (threadIdx.x & 63); b <= end; b += 64) sure = sure && table[b] >= 0 && table[b] < n_pages;
    sure = __ballot(!sure) == 0;
  }
};

// The granules of a list of pages of a sequence.
struct Chosen {
  const int *list, *table;
  int count, shift, n_pages, keys;
  __device__ __forceinline__ Granule operator()(int i) const {
    const int n = i >> (shift - kGranuleBits), last = (keys - 1) >> shift;
    const int b = n < count ? list[n] : -1;
    const int page = table[b < 0 ? 0 : b < last ? b : last];
    const bool there = b >= 0 && b <= last && page >= 0 && page < n_pages;
    return {there ? page : -1, there ? (b << shift) + ((i << kGranuleBits) & ((1 << shift) - 1)) : kNowhere};
  }
};

// The kernel's arguments, read again where they are asked for: the scalar registers do not hold all that a
// loop over keys and what is around it need, and what the compiler puts aside costs a read through a
// vector register each time.
template <typename A>
__device__ __forceinline__ const __attribute__((address_space(4))) A* arguments() {
  auto p = (const __attribute__((address_space(4))) A*)__builtin_amdgcn_kernarg_segment_ptr();
  if constexpr (A::kReadAgain) asm volatile("" : "+s"(p));
  return p;
}

// A granule's first rows of one key head, and how many of its rows are the sequence's (kWhole: all, and
// they are within 32-bit offsets).
constexpr int kWhole = kGranule + 1;
struct Spot {
  const void *k, *v;
  int rows, key;
};
struct __attribute__((aligned(16))) Place {
  size_t k, v;                         // 0: not there
};

__device__ __forceinline__ size_t read_lane(size_t v, int lane) {
  const u32 lo = __builtin_amdgcn_readlane((u32)v, lane), hi = __builtin_amdgcn_readlane((u32)(v >> 32), lane);
  return (size_t)hi << 32 | lo;
}
__device__ __forceinline__ Place read_lane(const Place& p, int lane) {
  return {read_lane(p.k, lane), read_lane(p.v, lane)};
}

// What copies the granules of key head h; V for 32 rows at a time, or for 16.
template <typename A, typename T, int DP, int PLACE_V(int) = place_v<DP>>
struct Store {
  int h, shift, keys;
  bool full;                           // D == DP
  GranuleCopy<T, DP, place_k<DP>> ko;
  GranuleCopy<T, DP, PLACE_V> vo;
  __device__ __forceinline__ Store(const A& a, int h, int shift, int keys, int lane)
      : h(h), shift(shift), keys(keys), full(a.D == DP), ko(a.K.token, a.D, lane), vo(a.V.token, a.D, lane) {}
  // May differ from lane to lane.
  __device__ __forceinline__ Place place(const Granule& g) const {
    const auto a = arguments<A>();
    const long long page = g.page, row = g.key & ((1 << shift) - 1);
    Place p;
    p.k = (size_t)(static_cast<const T*>(a->K.data) + page * a->K.page + row * a->K.token + h * a->K.head);
    p.v = (size_t)(static_cast<const T*>(a->V.data) + page * a->V.page + row * a->V.token + h * a->V.head);
    p.k = g.page < 0 ? 0 : p.k;
    p.v = g.page < 0 ? 0 : p.v;
    return p;
  }
  __device__ __forceinline__ bool quick() const {        // offsets of a granule's rows fit 32 bits
    const auto a = arguments<A>();
    return (unsigned long long)a->K.token < 1 << 24 && (unsigned long long)a->V.token < 1 << 24;
  }
  __device__ __forceinline__ Spot spot(const Place& p, int key, bool quick) const {
    Spot s;
    s.k = (const void*)p.k;
    s.v = (const void*)p.v;
    const int left = s.k ? keys - key : 0;
    s.rows = left >= kGranule && quick ? kWhole : left;
    s.key = key;
    return s;
  }
  __device__ __forceinline__ void copy_k(const Spot& s, u32 lds, bool once) const {
    if (s.rows == kWhole) ko.whole(static_cast<const T*>(s.k), lds, full, once);
    else ko.some(static_cast<const T*>(s.k), arguments<A>()->K.token, s.rows, lds);
  }
  __device__ __forceinline__ void copy_v(const Spot& s, u32 lds, bool once) const {
    if (s.rows == kWhole) vo.whole(static_cast<const T*>(s.v), lds, full, once);
    else vo.some(static_cast<const T*>(s.v), arguments<A>()->V.token, s.rows, lds);
  }
};

// n / d of small numbers (n < 2^22), by 1 / d.
__device__ __forceinline__ int quotient(int n, float inverse) { return (int)(((float)n + 0.5f) * inverse); }

// Where a tile's result goes: to O and lse, or, of a part of the keys, its sums in binary32.
template <typename T>
struct Target {
  T* O;                                // of the tile's first token and the key head's first query head
  float* lse;
  long long o_token, o_head;
  int Hq, group, first;                // first: row of the first token that the tile begins with
  float *po, *pml;                     // parts (or nullptr): row r at r * D and 2 * r
  int D;
  __device__ __forceinline__ void split(int r, int* token, int* head) const {
    *token = quotient(first + r, 1.0f / (float)group);
    *head = first + r - *token * group;
  }
};

constexpr int kTileKeys = 64, kManyRows = 128, kFewRows = 16, kFewKeys = 32;
template <int DP>
constexpr int kStages = DP <= 128 ? 2 : 1;
template <int DP>
struct Shared {
  static constexpr int kWaves = 4;
  union {
    uint8_t many[kStages<DP>][2][kTileKeys * 2 * DP];  // [stage][K, V]
    uint8_t few[4][2][kFewKeys * 2 * DP];              // [wavefront][K, V]
    float o[4][kFewRows][DP + 4];                      // parts of the output, rows 16 bytes apart in the banks
  };
  float ml[4][kFewRows][2];
  Place place[4][64];                                  // [wavefront][tile] (many)
};
// The same for few rows and one, two or four wavefronts.
template <int DP, int WAVES>
struct SharedFew {
  static constexpr int kWaves = WAVES;
  union {
    uint8_t few[WAVES][2][kFewKeys * 2 * DP];
    float o[WAVES][kFewRows][DP + 4];
  };
  float ml[WAVES][kFewRows][2];
};

// Zeros where a whole granule's copies leave LDS alone and products of K read it.
template <typename S>
__device__ __forceinline__ void clear(S& sh) {
  __syncthreads();
  u32x4* p = reinterpret_cast<u32x4*>(&sh);
  for (int i = threadIdx.x; i < (int)(sizeof(sh.few) / 16); i += 64 * S::kWaves) p[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
}

// Up to 128 rows by four wavefronts that share tiles of 64 keys, the next tile on its way while one is
// worked on; key tiles from lo to hi.  A wavefront copies one granule of each tile.  Every key that is read
// serves 128 rows, so what bounds it is what a wavefront issues, vector and matrix instructions hardly at the
// same time, as in the packed attention: 0.98 PFLOP/s for 4 x 1024 tokens over 8192 keys, 32/8 heads of 128
// (contiguous keys 0.98).
template <typename A, typename T, int DP, int DC, typename F>
__device__ __forceinline__ void attend_many(Shared<DP>& sh, const Store<A, T, DP>& store, Line where, const T* qp, int D,
                                            int sees, int all, int last, int lo, int hi, int rows, u32 flip, float c,
                                            float lift, F target) {
  constexpr int BYTES = kGranule * 2 * DP;             // of a granule in LDS
  constexpr int STAGES = kStages<DP>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool quick = store.quick();
  // The places of the wave's granules of 64 tiles, in LDS: a look at the table in every step is three
  // scalar loads in a row, which the matrix instructions behind them wait for (7 % of four times 1024 tokens
  // over 8192 keys).
  Place* const places = sh.place[wave];
  int base = 0;
  auto hold = [&](int i) {
    base = i;
    places[lane] = store.place(where(4 * (i + lane) + wave));
  };
  auto look = [&](int i) {
    if (i - base == 64) hold(i);
    return store.spot(read_lane(places[i - base], 0), (4 * i + wave) * kGranule, quick);
  };
  auto copy = [&](const Spot& s, int stage) {
    store.copy_k(s, lds_address(sh.many[stage][0]) + wave * BYTES, false);
    store.copy_v(s, lds_address(sh.many[stage][1]) + wave * BYTES, false);
  };
  Spot next = {nullptr, nullptr, 0, 0};
  if (lo < hi) {
    hold(lo);
    next = look(lo);
  }
  if (STAGES == 2 && lo < hi) {
    copy(next, 0);
    if (lo + 1 < hi) next = look(lo + 1);
  }
  Rows<T, DP, DC> w;
  w.start(qp, D, flip);
  w.addresses(lds_address(sh.many[0][0]), lds_address(sh.many[0][1]));
  where.look_over(lo * (kTileKeys / kGranule), hi * (kTileKeys / kGranule));
  for (int i = lo; i < hi; ++i) {
    const int stage = STAGES == 2 ? (i - lo) & 1 : 0;
    if (STAGES == 1) {
      __syncthreads();                                 // the last tile has been read
      copy(next, 0);
      if (i + 1 < hi) next = look(i + 1);
    }
    wait_copies();
    __syncthreads();
    if (STAGES == 2 && i + 1 < hi) copy(next, stage ^ 1);
    if (i * kTileKeys < last) {
      f32x16 s[2];
      u32 p[2][8];
      s[0] = w.scores(0);
      s[1] = w.scores(32);
      const bool masked = !where.sure || (i + 1) * kTileKeys > all;
      int key[4] = {0, 0, 0, 0};
      if (masked) {
#pragma unroll
        for (int g = 0; g < 4; ++g) key[g] = where.sure ? (4 * i + g) * kGranule : where(4 * i + g).key;
      }
      w.softmax(s, p, c, lift, masked, [&](int k) { return key[k / kGranule] + k % kGranule < sees; });
      w.values(0, p[0]);
      w.values(32, p[1]);
    }
    if (STAGES == 2) {
      if (i + 2 < hi) next = look(i + 2);
      w.move(stage ? -(int)sizeof(sh.many[0]) : (int)sizeof(sh.many[0]));
    }
  }
  const Target<T> to = target();
  int half = lane >> 5;
  if constexpr (DP > 128) asm volatile("" : "+v"(half)); // (or sums with it are held all the time, and spilled)

  const float l = w.l + other_half(w.l);
  const int r = wave * 32 + (lane & 31);
  if (r >= rows) return;
  // a row that sees no key: zeros, and -inf (its sums may hold 0 * NaN from values that others see)
  const bool none = no_weight(w.m, l);
  if (__ballot(none)) {                                // (hardly ever: no select in the ordinary way)
#pragma unroll
    for (int i = 0; i < DC / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) w.o[i][j] = none ? 0.f : w.o[i][j];
  }
  if (to.po) {
    float* po = to.po + (long long)r * to.D;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const int d = 32 * i + 2 * j + 4 * half;
        if (d < to.D) *reinterpret_cast<f32x4*>(po + d) = f32x4{w.o[i][j], w.o[i][j + 1], w.o[i][j + 2], w.o[i][j + 3]};
      }
    if (half == 0) *reinterpret_cast<f32x2*>(to.pml + 2 * r) = f32x2{w.m, l};
    return;
  }
  const float inv = none ? 0.f : 1.0f / l;
  int token, head;
  to.split(r, &token, &head);
  T* op = to.O + token * to.o_token + head * to.o_head;
#pragma unroll
  for (int i = 0; i < DC / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      const int d = 32 * i + 2 * j + 4 * half;
      if (d < to.D) {
        const float y[4] = {w.o[i][j] * inv, w.o[i][j + 1] * inv, w.o[i][j + 2] * inv, w.o[i][j + 3] * inv};
        store_floats<T, 4>(op + d, y);
      }
    }
  if (to.lse && half == 0) to.lse[(long long)token * to.Hq + head] = log_sum(w.m, l, c);
}

// 16 rows, for tiles of 32 keys: the heads of a single token's group.  Bound by memory, where tiles of 128
// rows would be by the zeros that they multiply: 16 tokens of 4000 to 32000 keys 195 us, as tiles of 128 rows
// 220; 256 tokens of 100 to 4000 366 and 406.
template <typename T, int DP, int DC>
struct Few16 {
  static constexpr int kRows = 16;
  Rows16<T, DP, DC> w;
  f32x4 s[2];
  u32x4 p;
  __device__ __forceinline__ void scores() {
    s[0] = w.scores(0);
    s[1] = w.scores(16);
  }
  template <typename F>
  __device__ __forceinline__ void softmax(float c, float lift, bool masked, F seen) {
    p = w.softmax(s, c, lift, masked, seen);
  }
  __device__ __forceinline__ void values() { w.values(p); }
  __device__ __forceinline__ float sum() const {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w.l), __float_as_uint(w.l), false, false);
    const float x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    return x + other_half(x);
  }
  // This lane's outputs of its row times `keep`, zeros if there is none.
  __device__ __forceinline__ void put(float* o, bool none, float keep) const {
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) {
      f32x4 y;
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = none ? 0.f : w.o[i][u] * keep;
      *reinterpret_cast<f32x4*>(o + 16 * i + 4 * ((threadIdx.x >> 4) & 3)) = y;
    }
  }
};
// Up to R::kRows rows: the wavefronts share out the tiles of 32 keys from lo to hi, each copying its own, K
// of the next while it works on V of this and the other way round; their parts are joined in LDS.
template <typename R, typename T, int DP, int DC, typename S, typename G, typename F, typename SH>
__device__ __forceinline__ void attend_few(SH& sh, const S& store, G where, const T* qp, int D,
                                           int sees, int all, int lo, int hi, int rows, bool once, u32 flip, float c,
                                           float lift, F target) {
  constexpr int WAVES = SH::kWaves, BYTES = kGranule * 2 * DP, COPIES = 2 * GranuleCopy<T, DP, place_k<DP>>::N;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u32 lk = lds_address(sh.few[wave][0]), lv = lds_address(sh.few[wave][1]);
  struct Two {
    Spot s[2];
  };
  // (as above; lanes hold the places of the granules of 32 tiles)
  const bool quick = store.quick();
  Place held = {};
  int held_key = 0, base = 0;
  auto hold = [&](int i) {
    base = i;
    const Granule g = where(2 * (i + WAVES * (lane >> 1)) + (lane & 1));
    held = store.place(g);
    held_key = g.key;
  };
  auto look = [&](int i) {
    if (i - base == 32 * WAVES) hold(i);
    const int from = (i - base) / WAVES * 2;
    return Two{{store.spot(read_lane(held, from), __builtin_amdgcn_readlane(held_key, from), quick),
                store.spot(read_lane(held, from + 1), __builtin_amdgcn_readlane(held_key, from + 1), quick)}};
  };
  auto copy_k = [&](const Two& t) {
    store.copy_k(t.s[0], lk, once);
    store.copy_k(t.s[1], lk + BYTES, once);
  };
  auto copy_v = [&](const Two& t) {
    store.copy_v(t.s[0], lv, once);
    store.copy_v(t.s[1], lv + BYTES, once);
  };
  int i = lo + wave;
  Two next = {};
  int key[2] = {0, 0};
  if (i < hi) {
    hold(i);
    next = look(i);
    copy_k(next);
    copy_v(next);
    key[0] = next.s[0].key;
    key[1] = next.s[1].key;
    if (i + WAVES < hi) next = look(i + WAVES);
  }
  R r;
  r.w.start(qp, D, flip);
  r.w.addresses(lk, lv);
  for (; i < hi; i += WAVES) {
    const bool more = i + WAVES < hi;
    // (copies arrive in order: all but the last COPIES, those of V, are there)
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
    r.scores();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K has been read
    if (more) copy_k(next);
    const bool masked = key[0] + kGranule > all || key[1] + kGranule > all;
    r.softmax(c, lift, masked, [&](int k) { return key[k / kGranule] + k % kGranule < sees; });
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
    else wait_copies();
    r.values();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V has been read
    if (more) {
      copy_v(next);
      key[0] = next.s[0].key;
      key[1] = next.s[1].key;
      if (i + 2 * WAVES < hi) next = look(i + 2 * WAVES);
    }
  }

  // join the wavefronts' parts: they refer to different maxima
  constexpr int ROWS = R::kRows;
  const int mine = lane & (ROWS - 1);
  const float m_own = r.w.m, l = r.sum();
  if (lane < ROWS) {
    sh.ml[wave][lane][0] = m_own;
    sh.ml[wave][lane][1] = l;
  }
  __syncthreads();                                       // (nobody reads K and V any more)
  float m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) m = fmaxf(m, sh.ml[v][mine][0]);
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const float mv = sh.ml[v][mine][0], lv = sh.ml[v][mine][1];
    if (!no_weight(mv, lv)) sum += lv * __builtin_amdgcn_exp2f((mv - m) * c);
  }
  // (a part in which a row sees no key is 0: its sums may hold 0 * NaN from values that others see)
  if (mine < rows) r.put(sh.o[wave][mine], no_weight(m_own, l), __builtin_amdgcn_exp2f((m_own - m) * c));
  __syncthreads();
  if (wave == 0 && lane < ROWS) {                        // for the threads that store a row
    sh.ml[0][lane][0] = m;
    sh.ml[0][lane][1] = sum;
  }
  __syncthreads();
  const Target<T> to = target();
  constexpr int QUADS = DC / 4;
  for (int e = threadIdx.x; e < rows * QUADS; e += 64 * WAVES) {
    const int r = e / QUADS, d = 4 * (e % QUADS);
    if (d >= to.D) continue;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < WAVES; ++v) y += *reinterpret_cast<const f32x4*>(&sh.o[v][r][d]);
    const float mr = sh.ml[0][r][0], lr = sh.ml[0][r][1];
    if (to.po) {
      *reinterpret_cast<f32x4*>(to.po + (long long)r * to.D + d) = y;
      if (d == 0) *reinterpret_cast<f32x2*>(to.pml + 2 * r) = f32x2{mr, lr};
    } else {
      const float inv = no_weight(mr, lr) ? 0.f : 1.0f / lr;
      const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
      int token, head;
      to.split(r, &token, &head);
      store_floats<T, 4>(to.O + token * to.o_token + head * to.o_head + d, z);
      if (to.lse && d == 0) to.lse[(long long)token * to.Hq + head] = log_sum(mr, lr, c);
    }
  }
  __syncthreads();                                       // (LDS is free for a next tile)
}

// Parts of a row: of the first one the sums are at ml and the values at o, the others' `step` rows behind
// each other from `gap` rows in front of it on.
struct Run {
  const float *ml, *o;
  long long step, gap;
  int count;
};

// Joins the parts of two runs for a row, by WAVES wavefronts that share them out.  A group of lanes has four
// outputs each of one part, as many parts at a time as there are groups, four times as many on their way, the
// first of them with the sums; weights are found before, a lane a part, by each wavefront for itself.
constexpr int kMaxPieces = 512;        // of a line
constexpr int kMaxParts = kMaxPieces + 4;
template <typename T, int WAVES>
__device__ __forceinline__ void join_row(float* weight, float (*sums)[TDQ_MAX_HEAD], const Run& a, const Run& b, int D,
                                         float scale_log2, T* op, float* lse) {
  constexpr int AHEAD = 4;
  const int lane = threadIdx.x & 63, wave = WAVES > 1 ? threadIdx.x >> 6 : 0, n = a.count + b.count;
  const int quads = D <= 32 ? 8 : D <= 64 ? 16 : D <= 128 ? 32 : 64;
  const int c = 4 * (lane & (quads - 1)), groups = 64 / quads * WAVES, group = lane / quads * WAVES + wave;
  auto row = [&](int i) {                                // of its run
    const bool first = i < a.count;
    const int at = first ? i : i - a.count;
    return at == 0 ? 0 : at * (first ? a.step : b.step) - (first ? a.gap : b.gap);
  };
  auto ml = [&](int i) { return *reinterpret_cast<const f32x2*>((i < a.count ? a.ml : b.ml) + 2 * row(i)); };
  auto value = [&](int i) { return *reinterpret_cast<const f32x4*>((i < a.count ? a.o : b.o) + row(i) * D + c); };
  f32x4 ahead[AHEAD];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + j * groups;
      ahead[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < D && i < n) ahead[j] = value(i);
    }
  };
  fetch(group);
  f32x2 own = {-INFINITY, 0.f};                          // of part `lane`
  if (lane < n) own = ml(lane);
  float m = own[0];
  for (int i = lane + 64; i < n; i += 64) m = fmaxf(m, ml(i)[0]);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  float l = 0.f;
  for (int i = lane; i < n; i += 64) {
    const f32x2 x = i == lane ? own : ml(i);
    // A part without keys is left out, marked by a negative weight.  One of nothing but NaN has the
    // same maximum of -inf, and its sum makes the row NaN; one whose weight rounds to 0 still counts,
    // as its values may not be finite.
    const bool none = no_weight(x[0], x[1]);
    const float f = x[1] != x[1] ? x[1] : __builtin_amdgcn_exp2f((x[0] - m) * scale_log2);
    weight[i] = none ? -1.f : f;
    if (!none) l = fmaf(x[1], f, l);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
  __builtin_amdgcn_wave_barrier();
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = group; i0 < n; i0 += AHEAD * groups) {
    if (i0 != group) fetch(i0);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + j * groups;
      const float f = i < n ? weight[i] : -1.f;
      if (!(f < 0.f)) y += ahead[j] * f;
    }
  }
  for (int d = 32; d >= quads; d >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] += __shfl_xor(y[i], d, 64);
  if constexpr (WAVES > 1) {
    if (lane < quads) *reinterpret_cast<f32x4*>(&sums[wave][c]) = y;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) y += *reinterpret_cast<const f32x4*>(&sums[w][c]);
  }
  const float inv = no_weight(m, l) ? 0.f : 1.0f / l;
  if (lane < quads && c < D) {
    const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
    store_floats<T, 4>(op + c, z);
    if (lse && lane == 0) *lse = log_sum(m, l, scale_log2);
  }
  __builtin_amdgcn_wave_barrier();
}

// The same for up to kFewParts parts, by the lanes that have the row's outputs, each for itself.
constexpr int kFewParts = 8;
template <typename T>
__device__ __forceinline__ void join_few(const Run& a, const Run& b, int c, int D, float scale_log2, T* op, float* lse) {
  const int n = a.count + b.count;
  f32x2 x[kFewParts];
  f32x4 v[kFewParts];
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    x[i] = f32x2{-INFINITY, 0.f};
    v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (i < n && c < D) {
      const bool first = i < a.count;
      const int at = first ? i : i - a.count;
      const long long row = at == 0 ? 0 : at * (first ? a.step : b.step) - (first ? a.gap : b.gap);
      x[i] = *reinterpret_cast<const f32x2*>((first ? a.ml : b.ml) + 2 * row);
      v[i] = *reinterpret_cast<const f32x4*>((first ? a.o : b.o) + row * D + c);
    }
  }
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) m = fmaxf(m, x[i][0]);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    // (what is left out and what is not: as above)
    const bool none = no_weight(x[i][0], x[i][1]);
    const float f = x[i][1] != x[i][1] ? x[i][1] : __builtin_amdgcn_exp2f((x[i][0] - m) * scale_log2);
    if (!none) {
      l = fmaf(x[i][1], f, l);
      y += v[i] * f;
    }
  }
  if (c < D) {
    const float inv = no_weight(m, l) ? 0.f : 1.0f / l;
    const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
    store_floats<T, 4>(op + c, z);
    if (lse && c == 0) *lse = log_sum(m, l, scale_log2);
  }
}
// A run as lane `from` of the wavefront has it.
__device__ __forceinline__ Run run_of(const Run& r, int from) {
  return Run{(const float*)__shfl((unsigned long long)r.ml, from, 64), (const float*)__shfl((unsigned long long)r.o, from, 64),
             __shfl(r.step, from, 64), __shfl(r.gap, from, 64), __shfl(r.count, from, 64)};
}

// ---------------------------------------------------------------------------
// whole sequences
// ---------------------------------------------------------------------------
// The work is laid out on a line, for every key head the same: first the prefixes (each with the rows of
// all its sequences), then the sequences with their own keys, of each its tiles of 128 rows, of each tile
// its keys.  A workgroup takes an equal piece of that line, whatever it holds of many short or parts of
// few long ones; a tile that lies in several pieces is joined by the second kernel.  Every workgroup finds
// the line's length and its own place on it from the lengths (a sum over them by all threads), so that
// nothing of the plan depends on the host, which does not know them.
//
// Keys and values that one tile reads stream past the caches (16 tokens of 4000 to 32000 keys 196 us, through
// them 218; 256 of 100 to 4000 366 and 402): what bounds single tokens is memory, 6.3 TB/s in the kernel.
struct PagedArgs {
  static constexpr bool kReadAgain = true;
  const void* Q;
  void* O;
  float* lse;
  Pages K, V;
  Sequences own, pre;                  // (pre.S = 0: none; pre.cu counts sequences)
  long long q_token, q_head, o_token, o_head;
  long long Tq;
  int Hq, Hk, group, D, causal;
  float scale_log2, lift;
  u32 flip;
  double per_group, half_tile;         // 1 / group, and half of the tokens of a tile
  int pieces;                          // most pieces of a line
  int cap;                             // rows of a part: as many as a tile may have
  int2* first_tile;                    // [prefixes + 1]: tiles of sequences and prefixes; of each those in front, first token
  int2* tiles;                         // [own_tiles + pre_tiles][Hk]: first piece of each, how many; sequences first
  long long own_tiles, pre_tiles;      // (room for so many)
  int4* place;                         // [Tq]: tile, row of it and sequence of a token's first row; or, if by_tile,
                                       // [own_tiles]: first token of a tile, rows of it in front, rows, sequence
  bool by_tile;                        // the second kernel joins by tiles
  float *part_o, *part_ml;             // [pieces Hk][2][cap]: of tiles that begin before a piece, and that end behind it
  float *whole_o, *whole_ml;           // with prefixes: [2][Tq Hq], of tiles of one (prefixes, sequences) in one piece
};

// With prefixes in the call every row of both kinds of items goes through the workspace in binary32 and is joined by
// the second kernel, those of sequences without a prefix too: 4 x 1024 tokens over 9024 keys of their own 595 us,
// with a prefix that belongs to nobody in the call 626, over 1024 of their own behind 8000 shared 642.

// What a tile takes beside its keys (its place, its first keys on their way, its stores), in tiles of 64 keys.
// us with 2, 4 and 8: 64 tokens behind a prefix 90, 87, 95; 16 questions behind three 32.6, 29.6, 31.5; others
// the same.  The shortest piece, us with 1, 2, 3, 4 and 6: those 16 questions 33.7, 31.2, 30.4, 29.4, 32.2; a
// prompt of 256 tokens 25.5, 23.8, 23.9, 30.6, 31.0; one token over 2000 keys 20.4, 18.8, 18.1, 17.8, 18.9; 8
// over 100 to 800 19.0, 18.4, 20.3, 20.7, 21.5.
constexpr int kTileCost = 4, kLeastPiece = 3;

// A prefix or a sequence: its rows, and its keys.
struct Item {
  int t0, end;                         // first token and the one behind the last
  int len, keys;                       // as given, and those that are within the line's room
  int ahead;                           // token i sees the keys up to i + ahead
  unsigned rows;
  int tiles, skip;                     // tiles, and how many of them see no key
  bool causal;

  // Cost of the first r tiles: kTileCost each, and the sum of what their last rows see in tiles of 64
  // keys, over skip < i <= r of 128 i / group + ahead (or ahead, where all see the same).
  __device__ __forceinline__ long long cost(const PagedArgs& a, int r) const {
    const int m = r > skip ? r - skip : 0;
    const double first = (double)(r - m), end = (double)r;
    double seen = (double)m * ahead;
    if (causal) seen += a.half_tile * (end * (end + 1.0) - first * (first + 1.0));
    return (long long)kTileCost * r + (long long)(seen * (1.0 / kTileKeys));
  }
  // Keys that a row sees.
  __device__ __forceinline__ int sees(const PagedArgs& a, unsigned row) const {
    const int e = (int)(((double)row + 0.5) * a.per_group) + ahead + 1;
    return e < 0 ? 0 : e < keys ? e : keys;
  }
};
__device__ __forceinline__ Item item_from(const PagedArgs& a, bool prefix, int t0, int end, int len) {
  const int room = (prefix ? a.pre.columns : a.own.columns) << a.own.shift, have = len < 0 ? 0 : len;
  Item x;
  x.t0 = t0;
  x.end = end;
  x.len = len;
  x.keys = have < room ? have : room;
  const int tokens = end > t0 ? end - t0 : 0;
  x.rows = (unsigned)tokens * (unsigned)a.group;
  x.tiles = (int)((x.rows + (unsigned)(kManyRows - 1)) / kManyRows);
  // (what sees everything: as if all its tokens stood at the end.  Token i is key have - tokens + i, also where
  // that is past the room; from the room's last key on a token sees all of them)
  x.causal = a.causal && !prefix;
  x.ahead = !x.causal ? x.keys : have - tokens < x.keys ? have - tokens : x.keys - 1;
  x.skip = 0;
  if (x.ahead < 0) {
    const long long none = (long long)-x.ahead * a.group / kManyRows;
    x.skip = none < x.tiles ? (int)none : x.tiles;
  }
  return x;
}
__device__ __forceinline__ Item item_of(const PagedArgs& a, int v) {
  const bool prefix = v < a.pre.S;
  int s = v - a.pre.S, next = s + 1;
  if (prefix) {
    s = start_of(a.pre.cu, v, a.own.S);
    next = start_of(a.pre.cu, v + 1, a.own.S);
  }
  return item_from(a, prefix, start_of(a.own.cu, s, a.Tq), start_of(a.own.cu, next, a.Tq),
                   prefix ? a.pre.len[v] : a.own.len[v - a.pre.S]);
}

// The tile of an item, and the place of it on the line.
struct Stretch {
  long long begin, end;
  int tiles;                           // of keys, one at least
  double each;                         // of them for one place
  __device__ __forceinline__ int at(long long x) const {   // first tile of keys behind a place
    if (x <= begin) return 0;
    if (x >= end) return tiles;
    const int n = (int)((double)(x - begin) * each);
    return n < tiles ? n : tiles - 1;
  }
};
__device__ __forceinline__ Stretch stretch_of(const PagedArgs& a, const Item& x, long long start, int r) {
  Stretch s;
  s.begin = start + x.cost(a, r);
  s.end = start + x.cost(a, r + 1);
  const unsigned behind = (unsigned)(r + 1) * kManyRows;
  const int n = x.sees(a, (behind < x.rows ? behind : x.rows) - 1);
  s.tiles = n > 0 ? (n + kTileKeys - 1) / kTileKeys : 1;
  s.each = (double)s.tiles / (double)(s.end - s.begin);
  return s;
}
__device__ __forceinline__ int pieces_of(const PagedArgs& a, long long total) {
  const long long n = total / kLeastPiece;
  return n < 1 ? 1 : n < a.pieces ? (int)n : a.pieces;
}
// The tile of all that workgroup k of n takes in a round of whole tiles.
__device__ __forceinline__ int tile_of_round(int round, int k, int n) { return round * n + (round & 1 ? n - 1 - k : k); }
// Whole tiles are no more than 1 + 1 / kSpare of a workgroup's share of the line.  us with none, 1 / 5, 1 / 3
// and 1 / 2: 4 x 1024 tokens over 8192 keys 665, 610, 610, 613; 16 times 100 to 600 tokens 512, 481, 549, 549;
// 40 times 1 to 500 733, 642, 643, 738; three long prompts of more tiles than workgroups 390, 399, 399, 400.
// Only up to 256 sequences and prefixes, which LDS has room for: 8 x 2048 tokens in a call of 256 sequences 414 us, of
// 257 436.
constexpr int kSpare = 5;

template <typename T, int DP, int DC>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 2 : 1))) void k_attend_pages(
    PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) Shared<DP> sh;
  __shared__ long long wave_sum[4];
  __shared__ int wave_tiles[4];
  // Of items, if there are no more: first token, end and length, where on the line, their first tile.
  __shared__ int3 known[256];
  __shared__ long long known_start[256];
  __shared__ int known_tile[256];
  __shared__ long long bounds[kMaxPieces + 1];           // where the pieces begin, and the last ends
  __shared__ long long wave_most[4], wave_slack[4];
  // Where the walk along the line is: in LDS, as the loops over keys leave no registers for it.
  __shared__ struct {
    long long start;                                     // where the item begins
    int item, tile0, r, pre_tiles;                       // item, its first tile, tile of it; tiles of prefixes
    int n, rounds, round;                                // pieces; rounds of whole tiles, and how many are done
  } walk;
  const int hk = (int)(blockIdx.x % (unsigned)a.Hk), k = (int)(blockIdx.x / (unsigned)a.Hk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // the line
  const int items = a.pre.S + a.own.S, share = (items + 255) / 256;
  const int v0 = tid * share < items ? tid * share : items, v1 = v0 + share < items ? v0 + share : items;
  long long mine = 0;
  int mine_tiles = 0;
  for (int v = v0; v < v1; ++v) {
    const Item x = item_of(a, v);
    mine += x.cost(a, x.tiles);
    mine_tiles += x.tiles;
    if (share == 1) known[v] = make_int3(x.t0, x.end, x.len);
  }
  long long upto = mine;
  int tiles_upto = mine_tiles;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(upto, d, 64);
    const int ot = __shfl_up(tiles_upto, d, 64);
    if (lane >= d) {
      upto += o;
      tiles_upto += ot;
    }
  }
  if (lane == 63) {
    wave_sum[wave] = upto;
    wave_tiles[wave] = tiles_upto;
  }
  __syncthreads();
  long long before = upto - mine, total = 0;
  int tiles_before = tiles_upto - mine_tiles, all_tiles = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) {
      before += wave_sum[w];
      tiles_before += wave_tiles[w];
    }
    total += wave_sum[w];
    all_tiles += wave_tiles[w];
  }
  const int n = pieces_of(a, total);
  if (total == 0 || k >= n) {
    if (blockIdx.x == 0 && tid == 0) a.first_tile[0] = make_int2(0, 0);
    return;
  }
  auto item = [&](int v) {
    if (share > 1) return item_of(a, v);
    const int3 x = known[v];
    return item_from(a, v < a.pre.S, x.x, x.y, x.z);
  };
  if (share == 1 && tid < items) {
    known_start[tid] = before;
    known_tile[tid] = tiles_before;
  }
  // The item of a tile (of all): the last that begins no later and has one.
  auto item_of_tile = [&](int j) {
    int v = 0;
    for (int count = items; count > 1;) {
      const int half = count / 2;
      if (known_tile[v + half] <= j) {
        v += half;
        count -= half;
      } else {
        count = half;
      }
    }
    return v;
  };
  // Whole tiles first, as long as they leave no workgroup with much more than its share: in round i
  // workgroup k takes tile i n + k, or in odd ones from the other end.  A cut tile's parts are 512 bytes a
  // row each way, so of tiles of few rows cuts cost little, and the plan more (256 single tokens 379 us,
  // without 368).
  const double per = (double)total / n;
  const long long each = (long long)per;
  int rounds = 0;
  long long load[2] = {0, 0};                            // of pieces 2 tid and 2 tid + 1
  if (share == 1 && a.Tq * a.group > (long long)kFewRows * all_tiles) {
    __syncthreads();
    for (int i = 0; (long long)(i + 1) * n <= all_tiles; ++i) {
      long long with[2], top = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int p = 2 * tid + u;
        with[u] = load[u];
        if (p < n) {
          const int j = tile_of_round(i, p, n), w = item_of_tile(j), r = j - known_tile[w];
          const Item x = item(w);
          with[u] += x.cost(a, r + 1) - x.cost(a, r);
        }
        top = with[u] > top ? with[u] : top;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const long long o = __shfl_xor(top, d, 64);
        top = o > top ? o : top;
      }
      if (lane == 0) wave_most[wave] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 4; ++w) top = wave_most[w] > top ? wave_most[w] : top;
      __syncthreads();
      if (top > each + each / kSpare) break;
      rounds = i + 1;
#pragma unroll
      for (int u = 0; u < 2; ++u) load[u] = with[u];
    }
  }
  if (rounds == 0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const long long at = (long long)((double)(2 * tid + u) * per);
      if (2 * tid + u < n) bounds[2 * tid + u] = at < total ? at : total;
    }
  } else {
    // The rest of the line is cut into pieces as long as what a workgroup's share is more than it has.
    long long rest = total;                              // where it begins
    if (rounds * n < all_tiles) {
      const int v = item_of_tile(rounds * n);
      rest = known_start[v] + item(v).cost(a, rounds * n - known_tile[v]);
    }
    long long slack[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) slack[u] = 2 * tid + u < n && load[u] < each ? each - load[u] : 0;
    long long sum = slack[0] + slack[1];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long o = __shfl_up(sum, d, 64);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_slack[wave] = sum;
    __syncthreads();
    long long all_slack = 0;
    sum -= slack[0] + slack[1];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) sum += wave_slack[w];
      all_slack += wave_slack[w];
    }
    // (whole numbers times the same factor: the bounds ascend; where there is no slack, the last has it all)
    const double stretch = all_slack > 0 ? (double)(total - rest) / (double)all_slack : 0.0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const long long at = rest + (long long)((double)sum * stretch);
      if (2 * tid + u < n) bounds[2 * tid + u] = at < total ? at : total;
      sum += slack[u];
    }
  }
  if (tid == 0) bounds[n] = total;
  __syncthreads();

  const long long from = bounds[k];
  for (int v = v0; v < v1; ++v) {
    long long next = before + mine;
    int tiles_next = tiles_before + mine_tiles;
    if (share > 1) {
      const Item x = item_of(a, v);
      next = before + x.cost(a, x.tiles);
      tiles_next = tiles_before + x.tiles;
    }
    if (before <= from && from < next) {
      walk.start = before;
      walk.item = v;
      walk.tile0 = tiles_before;
      walk.r = -1;
    }
    if (v == a.pre.S) walk.pre_tiles = tiles_before;
    if (blockIdx.x == 0 && v < a.pre.S) a.first_tile[v + 1] = make_int2(tiles_before, item(v).t0);
    before = next;
    tiles_before = tiles_next;
  }
  if (tid == 0) {
    walk.n = n;
    walk.rounds = rounds;
    walk.round = 0;
  }
  __syncthreads();

  if (blockIdx.x == 0 && tid == 0) a.first_tile[0] = make_int2(all_tiles - walk.pre_tiles, walk.pre_tiles);
  // (a piece of no length may lie within a tile: then it says so)
  if (rounds == 0 && from >= total) return;
  for (bool more = true; more;) {
    int v = __builtin_amdgcn_readfirstlane(walk.item), r = __builtin_amdgcn_readfirstlane(walk.r);
    int tile0 = __builtin_amdgcn_readfirstlane(walk.tile0);
    long long start = walk.start;
    const long long from = bounds[k], to = bounds[k + 1];
    const int n = __builtin_amdgcn_readfirstlane(walk.n), round = __builtin_amdgcn_readfirstlane(walk.round);
    const int pre_tiles = __builtin_amdgcn_readfirstlane(walk.pre_tiles);
    const bool whole = round < __builtin_amdgcn_readfirstlane(walk.rounds);
    if (whole) {
      const int j = tile_of_round(round, k, n);
      v = __builtin_amdgcn_readfirstlane(item_of_tile(j));
      tile0 = __builtin_amdgcn_readfirstlane(known_tile[v]);
      start = known_start[v];
      r = j - tile0;
    }
    Item x = item(v);
    if (r < 0) {                                         // the last tile that begins no later than the piece
      r = 0;
      for (int count = x.tiles; count > 1;) {
        const int half = count / 2;
        if (start + x.cost(a, r + half) <= from) {
          r += half;
          count -= half;
        } else {
          count = half;
        }
      }
      r = __builtin_amdgcn_readfirstlane(r);
    }
    const Stretch s = stretch_of(a, x, start, r);
    if (!whole && s.begin >= to) break;                  // (from here on the next piece's)
    const int lo = whole ? 0 : __builtin_amdgcn_readfirstlane(s.at(from));
    const int hi = __builtin_amdgcn_readfirstlane(whole ? s.tiles : s.at(to));
    const unsigned r0 = (unsigned)r * kManyRows;
    const int rows = __builtin_amdgcn_readfirstlane((int)(x.rows - r0 < kManyRows ? x.rows - r0 : kManyRows));
    const bool prefix = v < a.pre.S;
    const int line = prefix ? v : v - a.pre.S;
    const int token0 = __builtin_amdgcn_readfirstlane((int)(((double)r0 + 0.5) * a.per_group));
    const int first = __builtin_amdgcn_readfirstlane((int)(r0 - (unsigned)token0 * (unsigned)a.group));
    const int t0 = __builtin_amdgcn_readfirstlane(x.t0) + token0;
    const int keys = __builtin_amdgcn_readfirstlane(x.keys), tiles = __builtin_amdgcn_readfirstlane(s.tiles);
    const int ahead = __builtin_amdgcn_readfirstlane(x.ahead) + token0 + 1;   // of row r of the tile: + (first + r) / group
    // for the second kernel
    if (lo == 0 && lo < hi) {
      const long long tile = prefix ? a.own_tiles + tile0 + r : tile0 - pre_tiles + r;
      if (tid == 0 && tile < (prefix ? a.own_tiles + a.pre_tiles : a.own_tiles)) {
        // the last piece that the tile lies in: of those that begin in front of its end, and have some of it
        int last = k;
        if (!whole) {
          int beyond = n;
          while (beyond - last > 1) {
            const int half = (last + beyond) / 2;
            if (bounds[half] < s.end) last = half;
            else beyond = half;
          }
        }
        a.tiles[tile * a.Hk + hk] = make_int2(k, last - k + 1);
      }
      if (hk == 0 && !prefix && a.by_tile) {
        if (tid == 0 && tile < a.own_tiles) a.place[tile] = make_int4(t0, first, rows, line);
      } else if (hk == 0 && !prefix) {
        // tokens whose first row lies in the tile
        const int row = tid * a.group - first;
        if (row >= 0 && row < rows) a.place[t0 + tid] = make_int4(tile0 - pre_tiles + r, row, line, 0);
      }
    }
    if (lo >= hi && lo > 0 && lo < tiles && tid < rows) {
      // (no keys of the tile for this piece, though some for those before and behind)
      const long long slot = 2 * ((long long)k * a.Hk + hk);
      *reinterpret_cast<f32x2*>(a.part_ml + (slot * a.cap + tid) * 2) = f32x2{-INFINITY, 0.f};
    }
    // the next tile
    if (whole) {
      more = round + 1 < __builtin_amdgcn_readfirstlane(walk.rounds) || from < bounds[n];
    } else {
      more = s.end < to;
      if (++r >= x.tiles) {
        start += x.cost(a, x.tiles);
        tile0 += x.tiles;
        r = 0;
        while (more && ++v < items && item(v).tiles == 0) {
        }
        more = more && v < items;
      }
    }
    __syncthreads();                                     // (this tile has been read)
    if (tid == 0) {
      if (whole) {
        walk.round = round + 1;
      } else {
        walk.start = start;
        walk.item = v;
        walk.tile0 = tile0;
        walk.r = r;
      }
    }
    more = __builtin_amdgcn_readfirstlane((int)more) != 0;
    if (lo < hi) {
      const float per_group = (float)a.per_group;
      auto sees = [&](int row) {
        const int e = quotient(first + row, per_group) + ahead;
        return e < 0 ? 0 : e < keys ? e : keys;
      };
      const Line where = {prefix ? a.pre.table + line * a.pre.ld : a.own.table + line * a.own.ld, a.own.shift, a.own.n_pages,
                          keys, true};
      auto target = [&]() {
        const auto b = arguments<PagedArgs>();
        Target<T> to;
        to.O = static_cast<T*>(b->O) + t0 * b->o_token + (long long)hk * b->group * b->o_head;
        to.lse = b->lse ? b->lse + (long long)t0 * b->Hq + hk * b->group : nullptr;
        to.o_token = b->o_token;
        to.o_head = b->o_head;
        to.Hq = b->Hq;
        to.group = b->group;
        to.first = first;
        to.D = b->D;
        to.po = to.pml = nullptr;
        if (lo > 0 || hi < tiles) {
          const long long slot = 2 * ((long long)k * b->Hk + hk) + (lo > 0 ? 0 : 1);
          to.po = b->part_o + slot * b->cap * b->D;
          to.pml = b->part_ml + slot * b->cap * 2;
        } else if (b->pre.S > 0) {
          // (rows of a key head one after the other)
          const long long at = ((prefix ? 0 : b->Hk) + hk) * b->Tq * b->group + (long long)t0 * b->group + first;
          to.po = b->whole_o + at * b->D;
          to.pml = b->whole_ml + at * 2;
        }
        return to;
      };
      if (a.D < DC) clear(sh);
      const bool few = rows <= kFewRows;
      const int mine_row = few ? lane & 15 : wave * 32 + (lane & 31);
      const int row = mine_row < rows ? mine_row : rows - 1;
      const int token = quotient(first + row, per_group), head = first + row - token * a.group;
      const T* qp = static_cast<const T*>(a.Q) + (long long)(t0 + token) * a.q_token +
                    (long long)(hk * a.group + head) * a.q_head;
      const int end = __builtin_amdgcn_readfirstlane(sees(rows - 1));
      if (few) {
        const int all = __builtin_amdgcn_readfirstlane(sees(0));
        const int tiles = (end + kFewKeys - 1) / kFewKeys, stop = 2 * hi < tiles ? 2 * hi : tiles;
        int here = lane;                                 // (offsets computed here: held over the other loop, they
        if constexpr (DP <= 128) asm volatile("" : "+v"(here));   // are spilled there)
        const Store<PagedArgs, T, DP, place_v16<DP>> store(a, hk, a.own.shift, keys, here);
        attend_few<Few16<T, DP, DC>, T, DP, DC>(sh, store, where, qp, a.D, sees(row), all, 2 * lo, stop, rows, true,
                                                a.flip, a.scale_log2, a.lift, target);
      } else {
        const int from_row = wave * 32 < rows ? wave * 32 : rows - 1;
        const int last_row = wave * 32 + 31 < rows ? wave * 32 + 31 : rows - 1;
        const int last = wave * 32 < rows ? __builtin_amdgcn_readfirstlane(sees(last_row)) : 0;
        const int all = __builtin_amdgcn_readfirstlane(sees(from_row));
        const int tiles = (end + kTileKeys - 1) / kTileKeys, stop = hi < tiles ? hi : tiles;
        const Store<PagedArgs, T, DP> store(a, hk, a.own.shift, keys, lane);
        attend_many<PagedArgs, T, DP, DC>(sh, store, where, qp, a.D, sees(row), all, last, lo, stop, rows, a.flip,
                                          a.scale_log2, a.lift, target);
      }
    }
    if (more) __syncthreads();                           // (LDS is free, and the walk there)
  }
}

// Whether a sequence has a prefix, and that one's first tile and token.
struct Before {
  bool there;
  int2 first;
};
__device__ __forceinline__ Before prefix_of(const PagedArgs& a, int line) {
  const int lane = threadIdx.x & 63;
  Before b = {false, make_int2(0, 0)};
  if (a.pre.S <= 64) {                                   // all at once, a lane each
    int from = 0, to = 0;
    if (lane < a.pre.S) {
      from = start_of(a.pre.cu, lane, a.own.S);
      to = start_of(a.pre.cu, lane + 1, a.own.S);
      b.first = a.first_tile[1 + lane];
    }
    const unsigned long long mine = __ballot(line >= from && line < to);
    b.there = mine != 0;
    const int p = b.there ? __builtin_ctzll(mine) : 0;
    b.first.x = __builtin_amdgcn_readlane(b.first.x, p);
    b.first.y = __builtin_amdgcn_readlane(b.first.y, p);
  } else {
    const int p = last_at_most(a.pre.S, line, [&](int i) { return start_of(a.pre.cu, i, a.own.S); });
    b.there = line >= start_of(a.pre.cu, p, a.own.S) && line < start_of(a.pre.cu, p + 1, a.own.S);
    b.first = a.first_tile[1 + p];
  }
  return b;
}

// A row as its lanes have it: token and head, of key head hk and in its group, and its row of a tile in the
// pieces from own.x on, own.y of them.
struct RowOf {
  bool real;
  long long t;
  int h, hk, e, row;
  int2 own;
};
// Joins 64 / quads rows at a time, the lanes of each with four outputs; those of many parts one by one.
template <typename T, int WAVES>
__device__ __forceinline__ void join_rows(const PagedArgs& a, float* weight, float (*sums)[TDQ_MAX_HEAD], const RowOf& x,
                                          const Before& before, const int2& tiles, int quads) {
  const int lane = threadIdx.x & 63, c = 4 * (lane & (quads - 1));
  const long long pre_at = (x.t - before.first.y) * a.group + x.e, of = before.first.x + pre_at / kManyRows;
  const int pre_row = (int)(pre_at % kManyRows);
  int2 pre = make_int2(0, 0);
  if (x.real && before.there && pre_at >= 0 && of < tiles.y && of < a.pre_tiles && pre_row < a.cap)
    pre = a.tiles[(a.own_tiles + of) * a.Hk + x.hk];
  const bool wanted = x.real && (x.own.y > 1 || a.pre.S > 0);   // (else its one piece has written the output)
  if (__ballot(wanted) == 0) return;
  const long long step = 2ll * a.Hk * a.cap, whole = x.hk * a.Tq * a.group + x.t * a.group + x.e;
  // (parts of a tile: the first ends behind its piece, the others begin in front of theirs)
  auto run = [&](const int2& d, int row, long long whole) {
    const long long at = ((2ll * d.x * a.Hk + 2 * x.hk) + 1) * a.cap + row;
    return d.y == 1 ? Run{a.whole_ml + 2 * whole, a.whole_o + whole * a.D, 0, 0, 1}
                    : Run{a.part_ml + 2 * at, a.part_o + at * a.D, step, a.cap, d.y};
  };
  const Run p = run(pre, pre_row, whole), y = run(x.own, x.row, a.Tq * a.Hq + whole);
  T* op = static_cast<T*>(a.O) + x.t * a.o_token + x.h * a.o_head;
  float* lse = a.lse ? a.lse + x.t * a.Hq + x.h : nullptr;
  if (__ballot(wanted && p.count + y.count > kFewParts) == 0) {
    if (wanted && (WAVES == 1 || threadIdx.x < 64)) join_few<T>(p, y, c, a.D, a.scale_log2, op, lse);
    return;
  }
  for (int i = 0; i < 64; i += quads) {
    if (!__shfl((int)wanted, i, 64)) continue;
    join_row<T, WAVES>(weight, sums, run_of(p, i), run_of(y, i), a.D, a.scale_log2,
                       (T*)__shfl((unsigned long long)op, i, 64), (float*)__shfl((unsigned long long)lse, i, 64));
  }
}
__device__ __forceinline__ int quads_of(int D) { return D <= 32 ? 8 : D <= 64 ? 16 : D <= 128 ? 32 : 64; }

// Joins the tiles that lie in several pieces, and prefixes with sequences: calls of few rows, a wavefront or a
// workgroup a row.  What bounds it is a chain of four loads (the token's place, its tile, the sums, the values),
// 5 us for single tokens.
template <typename T, int WAVES>
__global__ __launch_bounds__(256, 4) void k_join_pages(PagedArgs a, int chunks) {
  __shared__ float weight[4][kMaxParts];
  __shared__ __attribute__((aligned(16))) float sums[WAVES][TDQ_MAX_HEAD];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const long long t = id / chunks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = (int)(id % chunks) * (4 / WAVES) + (WAVES > 1 ? 0 : wave);
  if (t >= a.Tq || h >= a.Hq) return;
  // (all on their way at once; what lies there is looked at if the token is one of a sequence)
  const int begin = start_of(a.own.cu, 0, a.Tq), end = start_of(a.own.cu, a.own.S, a.Tq);
  const int2 tiles = a.first_tile[0];                    // of sequences, of prefixes
  const int4 place = a.place[t];
  Before before = {false, make_int2(0, 0)};
  if (a.pre.S > 0) before = prefix_of(a, __builtin_amdgcn_readfirstlane(place.z));
  if (t < begin || t >= end || place.y < 0 || place.x < 0) return;
  const int quads = quads_of(a.D);
  RowOf x;
  x.t = t;
  x.h = h;
  x.hk = quotient(h, (float)a.per_group);
  x.e = h - x.hk * a.group;
  const long long own_row = (long long)place.y + x.e, tile = place.x + own_row / kManyRows;
  x.row = (int)(own_row % kManyRows);
  x.real = lane < quads && tile < tiles.x && tile < a.own_tiles && x.row < a.cap;
  x.own = make_int2(0, 1);
  if (x.real) x.own = a.tiles[tile * a.Hk + x.hk];
  join_rows<T, WAVES>(a, weight[wave], sums, x, before, tiles, quads);
}

// The same for calls of many rows: a workgroup one of the shares of a tile, which ends at once where the tile
// lies in one piece.  Bound by the parts, 67 MB of 2257 tokens.
template <typename T>
__global__ __launch_bounds__(256, 4) void k_join_tiles(PagedArgs a, int shares) {
  __shared__ float weight[4][kMaxParts];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int hk = (int)(id % a.Hk), part = (int)(id / a.Hk % shares);
  const long long tile = id / a.Hk / shares;
  if (tile >= a.own_tiles) return;
  const int2 tiles = a.first_tile[0];
  const int2 own = a.tiles[tile * a.Hk + hk];
  if (tile >= tiles.x || (own.y <= 1 && a.pre.S == 0)) return;
  const int4 span = a.place[tile];                       // first token, its row in front, rows, sequence
  Before before = {false, make_int2(0, 0)};
  if (a.pre.S > 0) before = prefix_of(a, __builtin_amdgcn_readfirstlane(span.w));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quads = quads_of(a.D), share = kManyRows / 4 / shares, r0 = (part * 4 + wave) * share;
  for (int i = 0; i < share && r0 + i < span.z; i += 64 / quads) {
    const int row = r0 + i + lane / quads;
    RowOf x;
    x.real = i + lane / quads < share && row < span.z;
    const int at = span.y + (x.real ? row : 0), token = quotient(at, (float)a.per_group);
    x.t = span.x + token;
    x.hk = hk;
    x.e = at - token * a.group;
    x.h = hk * a.group + x.e;
    x.row = row;
    x.own = own;
    join_rows<T, 1>(a, weight[wave], nullptr, x, before, tiles, quads);
  }
}

// Pieces for each key head's line: a workgroup each, as many as run at a time.  us with half, as many and
// twice: 16 tokens of 4000 to 32000 keys 194, 196, 201; 64 behind a prefix 119, 89, 105; 4 prompts' parts of
// 300 to 1024 tokens 449, 302, 327.
static int paged_pieces(int Hk, int D) {
  const int at_a_time = D <= 128 ? 512 : 256;
  return at_a_time / Hk > 0 ? at_a_time / Hk : 1;
}

// Rows of a call that four wavefronts each join: few rows have parts of up to 512 pieces, and wait for them.  us
// by one and by four: 8 rows over 100000 keys 88 and 43, of a prefix of 21354 35 and 25, 64 rows over 10947 26 and
// 21, 512 over 4000 to 32000 196 both; 1824 rows behind 11399 31 and 35, 2048 over 100 to 1000 38 and 41.
constexpr int kWholeRows = 512;

// More rows than this are joined by tiles, others one by one.  us by rows and by tiles: 8 x 2048 tokens of 32 heads
// 499 and 366, 4 x 1024 620 and 587, four prompts' parts of 355 to 1024 301 and 289; 512 tokens of 301 keys 131
// and 135, 64 times 5 244 and 249, one prompt of 256 23.2 and 24.5.
static bool by_tile(long long Tq, int Hq) { return Tq * Hq > 16384; }

struct PagedLayout {
  size_t tiles, place, ml, o, whole_ml, whole_o, total;  // (the first tiles at 0)
  int pieces, cap;
  long long own_tiles, pre_tiles;                        // at most
};
static PagedLayout paged_layout(long long Tq, int S, int prefixes, int Hq, int Hk, int D) {
  PagedLayout l;
  const long long rows = Tq * (Hq / Hk);
  l.cap = (int)(rows < kManyRows ? rows : kManyRows);
  l.pieces = paged_pieces(Hk, D);
  const size_t parts = 2ull * l.pieces * Hk * l.cap, whole = prefixes > 0 ? 2ull * Tq * Hq : 0;
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  l.own_tiles = rows / kManyRows + S;
  l.tiles = up((size_t)(prefixes + 1) * sizeof(int2));
  l.pre_tiles = prefixes > 0 ? rows / kManyRows + prefixes : 0;
  l.place = l.tiles + up((size_t)(l.own_tiles + l.pre_tiles) * Hk * sizeof(int2));
  l.ml = l.place + up((size_t)(by_tile(Tq, Hq) ? l.own_tiles : Tq) * sizeof(int4));
  l.o = l.ml + up(parts * 2 * sizeof(float));
  l.whole_ml = l.o + up(parts * D * sizeof(float));
  l.whole_o = l.whole_ml + up(whole * 2 * sizeof(float));
  l.total = l.whole_o + up(whole * D * sizeof(float));
  return l;
}
size_t paged_workspace(long long Tq, int S, int prefixes, int Hq, int Hk, int D) {
  return paged_layout(Tq, S, prefixes, Hq, Hk, D).total;
}

static Pages pages_of(const tdq_pages* p) { return {p->data, p->page, p->token, p->head}; }
static void scale_of(float scale, tdq_dtype dt, float* scale_log2, float* lift, u32* flip) {
  const double c = fabs((double)scale) * 1.44269504088896340736;
  *scale_log2 = c > 1e-30 ? (float)c : 1e-30f;           // (a masked score stays -inf)
  *lift = (dt == TDQ_F16 ? kLift<_Float16> : kLift<__bf16>) / *scale_log2;
  *flip = scale < 0.f ? 0x80008000u : 0u;                // (Q is negated)
}

// Kernels for a head of D elements: rows of LDS of a power of two, products of a multiple of 32.
#define TDQ_BY_HEAD(F, T)              \
  do {                                 \
    if (D <= 32) F(T, 32, 32);         \
    else if (D <= 64) F(T, 64, 64);    \
    else if (D <= 96) F(T, 128, 96);   \
    else if (D <= 128) F(T, 128, 128); \
    else if (D <= 192) F(T, 256, 192); \
    else F(T, 256, 256);               \
  } while (0)

hipError_t launch_paged(const tdq_heads* Q, const tdq_pages* K, const tdq_pages* V, tdq_dtype dt, long long Tq,
                        const tdq_sequences* seq, const tdq_sequences* prefix, int Hq, int Hk, int D, float scale,
                        bool causal, const tdq_heads* O, float* lse, void* workspace, hipStream_t st) {
  PagedArgs a;
  a.Q = Q->data;
  a.O = O->data;
  a.lse = lse;
  a.K = pages_of(K);
  a.V = pages_of(V);
  a.own = sequences_of(seq);
  if (prefix) {
    a.pre = sequences_of(prefix);
  } else {
    a.pre = a.own;
    a.pre.S = 0;
  }
  a.q_token = Q->token;
  a.q_head = Q->head;
  a.o_token = O->token;
  a.o_head = O->head;
  a.Tq = Tq;
  a.Hq = Hq;
  a.Hk = Hk;
  a.group = Hq / Hk;
  a.D = D;
  a.causal = causal;
  scale_of(scale, dt, &a.scale_log2, &a.lift, &a.flip);
  a.per_group = 1.0 / a.group;
  a.half_tile = kManyRows * 0.5 / a.group;
  const PagedLayout l = paged_layout(Tq, seq->S, a.pre.S, Hq, Hk, D);
  a.pieces = l.pieces;
  a.cap = l.cap;
  char* w = static_cast<char*>(workspace);
  a.first_tile = reinterpret_cast<int2*>(w);
  a.tiles = reinterpret_cast<int2*>(w + l.tiles);
  a.place = reinterpret_cast<int4*>(w + l.place);
  a.by_tile = by_tile(Tq, Hq);
  a.own_tiles = l.own_tiles;
  a.pre_tiles = l.pre_tiles;
  a.part_ml = reinterpret_cast<float*>(w + l.ml);
  a.part_o = reinterpret_cast<float*>(w + l.o);
  a.whole_ml = reinterpret_cast<float*>(w + l.whole_ml);
  a.whole_o = reinterpret_cast<float*>(w + l.whole_o);
  const dim3 grid((unsigned)(a.pieces * Hk));
#define TDQ_PAGED(T, DP, DC) hipLaunchKernelGGL((k_attend_pages<T, DP, DC>), grid, dim3(256), 0, st, a)
  if (dt == TDQ_F16) TDQ_BY_HEAD(TDQ_PAGED, _Float16);
  else TDQ_BY_HEAD(TDQ_PAGED, __bf16);
#undef TDQ_PAGED
  // (of tiles with few rows one.  us with one and four: 4096 tokens over 301 keys 1010 and 1067, 600 times 4
  // behind a prefix 315 and 384; 16 times 100 to 600 tokens 489 and 470)
  const int shares = Tq * a.group >= 64ll * seq->S ? 4 : 1;
#define TDQ_JOIN(T)                                                                                                 \
  do {                                                                                                              \
    if (a.by_tile)                                                                                                  \
      hipLaunchKernelGGL((k_join_tiles<T>), two_axes(l.own_tiles * Hk * shares), dim3(256), 0, st, a, shares);      \
    else if (Tq * Hq <= kWholeRows)                                                                                 \
      hipLaunchKernelGGL((k_join_pages<T, 4>), two_axes(Tq * Hq), dim3(256), 0, st, a, Hq);                         \
    else                                                                                                            \
      hipLaunchKernelGGL((k_join_pages<T, 1>), two_axes(Tq * ((Hq + 3) / 4)), dim3(256), 0, st, a, (Hq + 3) / 4);   \
  } while (0)
  if (dt == TDQ_F16) TDQ_JOIN(_Float16);
  else TDQ_JOIN(__bf16);
#undef TDQ_JOIN
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// chosen pages
// ---------------------------------------------------------------------------
// Every token and key head has a list of pages of its own, so a tile has the group's rows and no more;
// its pages are shared out to `splits` workgroups, and in each to four wavefronts, or, of many lists, two or one.
// Pages of single tokens are read once, at 6.2 TB/s (32 tokens, 64 pages of 64 keys, 8 heads of 128: 87 us); those
// of a prompt's tokens come from the caches, at 14 TB/s (401 tokens, 16 pages, 4 heads of 64: 28 us).
struct ChosenArgs {
  static constexpr bool kReadAgain = false;
  const void* Q;
  void* O;
  float* lse;
  Pages K, V;
  Sequences seq;
  const int* chosen;                   // [Tq Hk, count]
  long long q_token, q_head, o_token, o_head;
  long long Tq;
  int Hq, Hk, group, D, causal, count;
  float scale_log2, lift;
  u32 flip;
  int splits, tiles;                   // tiles of 16 rows of a group
  float *part_o, *part_ml;             // [splits][Tq Hq]
};

template <typename T, int DP, int DC, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 2 : 1))) void k_attend_chosen(
    ChosenArgs a) {
  __shared__ __attribute__((aligned(1024))) SharedFew<DP, WAVES> sh;
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int hk = (int)(id % a.Hk), split = (int)(id / a.Hk % a.splits);
  const long long rest = id / a.Hk / a.splits;
  const int tile = (int)(rest % a.tiles);
  const long long t = rest / a.tiles;
  if (t >= a.Tq) return;
  const Sequences& q = a.seq;
  const Owner o = owner_of(q, t, a.Tq);
  const int s = o.seq, from = o.from, to = o.to, keys = __builtin_amdgcn_readfirstlane(keys_in(q, o.len));
  if (t < from || t >= to) return;
  const int sees = __builtin_amdgcn_readfirstlane(keys_seen(q, o.len, to, t, a.causal));
  const int left = a.group - tile * kFewRows, rows = left < kFewRows ? left : kFewRows;
  const int lane = threadIdx.x & 63, row = (lane & 15) < rows ? lane & 15 : rows - 1;
  const int h0 = hk * a.group + tile * kFewRows;
  const int* list = a.chosen + (t * a.Hk + hk) * a.count;
  const Store<ChosenArgs, T, DP, place_v16<DP>> store(a, hk, q.shift, keys, lane);
  Target<T> target;
  target.O = static_cast<T*>(a.O) + t * a.o_token + h0 * a.o_head;
  target.lse = a.lse ? a.lse + t * a.Hq + h0 : nullptr;
  target.o_token = a.o_token;
  target.o_head = a.o_head;
  target.Hq = a.Hq;
  target.group = kFewRows;                            // (all rows are heads of one token)
  target.first = 0;
  target.D = a.D;
  target.po = target.pml = nullptr;
  if (a.splits > 1) {
    // (rows of a split one after the other)
    const long long at = (split * a.Tq + t) * a.Hq + h0;
    target.po = a.part_o + at * a.D;
    target.pml = a.part_ml + 2 * at;
  }
  int used = 0;                                          // the list up to its last page that is named
  for (int i = lane; i < a.count; i += 64) used = list[i] >= 0 ? i + 1 : used;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) used = max(used, __shfl_xor(used, d, 64));
  used = __builtin_amdgcn_readfirstlane(used);
  const int tiles = sees > 0 ? (int)((((long long)used << q.shift) + kFewKeys - 1) / kFewKeys) : 0;
  const int share = (tiles + a.splits - 1) / a.splits;
  const int lo = split * share < tiles ? split * share : tiles, hi = lo + share < tiles ? lo + share : tiles;
  Chosen where = {list, q.table + s * q.ld, used, q.shift, q.n_pages, keys};
  if (a.D < DC) clear(sh);
  attend_few<Few16<T, DP, DC>, T, DP, DC>(sh, store, where,
                                          static_cast<const T*>(a.Q) + t * a.q_token + (h0 + row) * a.q_head, a.D, sees,
                                          sees, lo, hi, rows, to - from == 1, a.flip, a.scale_log2, a.lift,
                                          [&] { return target; });
}

template <typename T>
__global__ __launch_bounds__(256, 4) void k_join_chosen(ChosenArgs a) {
  __shared__ float weight[4][kMaxParts];
  const long long row = 4 * (blockIdx.x + (long long)blockIdx.y * gridDim.x) + (threadIdx.x >> 6);
  if (row >= a.Tq * a.Hq) return;
  const long long t = row / a.Hq;
  const int h = (int)(row - t * a.Hq);
  const Sequences& q = a.seq;
  const int s = last_at_most(q.S, t, [&](int i) { return start_of(q.cu, i, a.Tq); });
  if (t < start_of(q.cu, s, a.Tq) || t >= start_of(q.cu, s + 1, a.Tq)) return;
  join_row<T, 1>(weight[threadIdx.x >> 6], nullptr, Run{}, Run{a.part_ml + 2 * row, a.part_o + row * a.D, a.Tq * a.Hq, 0, a.splits},
              a.D, a.scale_log2,
              static_cast<T*>(a.O) + t * a.o_token + h * a.o_head, a.lse ? a.lse + row : nullptr);
}

// Workgroups for the chip, as long as each has 256 keys.  us with 512, 1024 and 2048 of them: 32 tokens of 4096
// keys 91, 92, 96; 128 tokens 330, 330, 344.  With 128, 256 and 512 keys at least: one token 14.8, 14.4, 15.8,
// four 27, 22, 21.
static int chosen_splits(long long Tq, int Hq, int Hk, int page_size, int count) {
  const long long base = Tq * Hk * ((Hq / Hk + kFewRows - 1) / kFewRows), most = (long long)count * page_size / 256;
  long long n = 512 / base;
  if (n > most) n = most;
  if (n > 64) n = 64;
  return n > 1 ? (int)n : 1;
}
// Wavefronts of a list: four, as long as there is room for all lists at a time (LDS: 256 CUs, 256 / D workgroups on
// each); up to three times as many two; of more one: no keys too few for four, no parts to join, no waiting for
// the slowest.  us by four / two / one wavefronts, lists of 96 and of 1024 keys:
//   heads of 64   512 lists  11 /  - / 10 and  14 / 21 / 31   1604 lists 12 / 11 /  - and 28 / 27 / 36
//                3200 lists  21 /  - / 11 and  48 /  - / 45  12800 lists 64 /  - / 29 and 165 / - / 138
//   heads of 128  512 lists  11 / 11 /  - and  19 / 25 /  -   1024 lists 15 / 11 / 11 and 33 / 27 / 41
//                1440 lists  20 / 16 /  - and  46 / 47 /  -   6400 lists 69 /  - / 30 and 180 / - / 136
//   heads of 256  256 lists  11 / 11 /  - and  34 / 28 /  -   1024 lists 32 /  - / 15 and 85 / -  / 68
static int chosen_waves(long long lists, int D) {
  const int row = D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256;
  return lists * row <= 256 * 256 ? 4 : lists * row < 3 * 256 * 256 ? 2 : 1;
}
static size_t chosen_ml_bytes(long long Tq, int Hq, int splits) {
  return ((size_t)Tq * Hq * splits * 2 * sizeof(float) + 255) & ~(size_t)255;
}
size_t chosen_workspace(long long Tq, int Hq, int Hk, int D, int page_size, int count) {
  const int splits = chosen_splits(Tq, Hq, Hk, page_size, count);
  return splits > 1 ? chosen_ml_bytes(Tq, Hq, splits) + (size_t)Tq * Hq * splits * D * sizeof(float) : 0;
}

hipError_t launch_chosen(const tdq_heads* Q, const tdq_pages* K, const tdq_pages* V, tdq_dtype dt, long long Tq,
                         const tdq_sequences* seq, int Hq, int Hk, int D, float scale, bool causal, const int* chosen,
                         int count, const tdq_heads* O, float* lse, void* workspace, hipStream_t st) {
  ChosenArgs a;
  a.Q = Q->data;
  a.O = O->data;
  a.lse = lse;
  a.K = pages_of(K);
  a.V = pages_of(V);
  a.seq = sequences_of(seq);
  a.chosen = chosen;
  a.q_token = Q->token;
  a.q_head = Q->head;
  a.o_token = O->token;
  a.o_head = O->head;
  a.Tq = Tq;
  a.Hq = Hq;
  a.Hk = Hk;
  a.group = Hq / Hk;
  a.D = D;
  a.causal = causal;
  a.count = count;
  scale_of(scale, dt, &a.scale_log2, &a.lift, &a.flip);
  a.splits = chosen_splits(Tq, Hq, Hk, seq->page_size, count);
  a.tiles = (a.group + kFewRows - 1) / kFewRows;
  a.part_ml = static_cast<float*>(workspace);
  a.part_o = a.splits > 1
                 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + chosen_ml_bytes(Tq, Hq, a.splits))
                 : nullptr;
  const dim3 grid = two_axes(Tq * a.tiles * a.splits * Hk);
  const int waves = chosen_waves(Tq * a.tiles * a.splits * Hk, D);
#define TDQ_CHOSEN(T, DP, DC)                                                                             \
  do {                                                                                                    \
    if (waves == 1) hipLaunchKernelGGL((k_attend_chosen<T, DP, DC, 1>), grid, dim3(64), 0, st, a);        \
    else if (waves == 2) hipLaunchKernelGGL((k_attend_chosen<T, DP, DC, 2>), grid, dim3(128), 0, st, a);  \
    else hipLaunchKernelGGL((k_attend_chosen<T, DP, DC, 4>), grid, dim3(256), 0, st, a);                  \
  } while (0)
  if (dt == TDQ_F16) TDQ_BY_HEAD(TDQ_CHOSEN, _Float16);
  else TDQ_BY_HEAD(TDQ_CHOSEN, __bf16);
#undef TDQ_CHOSEN
  if (a.splits > 1) {
    const dim3 join = two_axes((Tq * Hq + 3) / 4);
    if (dt == TDQ_F16) hipLaunchKernelGGL((k_join_chosen<_Float16>), join, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_join_chosen<__bf16>), join, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}
#undef TDQ_BY_HEAD

}  // namespace tdq
