// Device skeleton of the plane family: products that meet in a plane of
// scores, which never leaves the registers.
//
// The plane has an owned and a streamed axis.  A wave owns 32 indices of the
// owned axis, one per lane pair (lane & 31), and walks over the streamed axis
// in tiles of TS.  For every subtile of 32 streamed indices:
//   scores  x_p = A_p . B_p       A_p: streamed rows (LDS), B_p: owned rows (registers)
//   plane   X_o = f(x, vectors)   the kernel's own elementwise expression
//   outputs acc_o += W_o^T . X_o  W_o: streamed rows (LDS)
// The 32 x 32 matrix instructions put the streamed index in an accumulator's
// register and the owned index in its lane, which is the layout that the
// second product takes as its right operand (for 16-bit types two groups of
// four registers make one operand of eight; the left operand's rows are read
// in the same order).  So the plane needs no pass through LDS and no shuffle.
// With a softmax the row maximum and sum run along (one pass over the data);
// the reference of the exponentials only moves when the maximum has grown by
// more than kLazy, which keeps the rescaling of the accumulators rare and the
// exponentials below 2^8 (2^15 with fp16's factor: no overflow);
// the results are brought to the true maximum at the end.
//
// Tiles whose mask is 0 for every pair are never loaded: the mask's value
// range over a tile follows from the ranges of its vectors (interval
// arithmetic), and the tiles with work are listed first.  The same ranges tell
// tiles whose mask is 0 for no pair, which skip it.
//
// P (generated) describes the kernel; see the constants and functions used.

typedef int i32x4 __attribute__((ext_vector_type(4)));

static constexpr float kLog2e = 1.4426950408889634f;
static constexpr float kLazy = 5.5f;  // natural units: 2^8
static constexpr int kListCap = 2048;

template <typename T> struct is_f16 {
  static constexpr bool value = false;
};
template <> struct is_f16<f16> {
  static constexpr bool value = true;
};

template <typename T> struct Mma;
template <> struct Mma<f16> {
  static constexpr int VL = 8, KU = 16;  // elements of a 16-byte vector; contraction covered by one fragment
  typedef f16x8 Frag;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<bf16> {
  static constexpr int VL = 8, KU = 16;
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
  static constexpr int VL = 4, KU = 8;
  typedef f32x4 Frag;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

constexpr int round_up(int x, int m) { return (x + m - 1) / m * m; }

// Geometry of a policy's LDS.
template <class P> struct Geo {
  typedef typename P::T T;
  static constexpr int VL = Mma<T>::VL, KU = Mma<T>::KU;
  static constexpr int NT = P::NW * 64;                 // threads of the workgroup
  static constexpr int GT = P::WSPLIT ? 64 : NT;        // threads that share a streamed tile
  static constexpr int NG = P::WSPLIT ? P::NW : 1;      // such groups
  static constexpr int OT = P::WSPLIT ? 32 : 32 * P::NW;  // owned indices of the workgroup
  static constexpr bool DMA = P::DMA;                   // tiles go straight to LDS
  static constexpr int NSUB = P::TS / 32;
  static constexpr int width(int t) { return round_up(P::sw(t), 32); }
  // Rows lie back to back; a row's 16-byte chunk c is stored at chunk c ^ swz(row).
  // The score products read one chunk of 32 rows at a time, the output products
  // 64 consecutive bytes of four rows (transposed); with the chunks of the 16
  // rows that share their address modulo the 256 bytes of all banks permuted
  // like this, neither meets a bank twice.
  static constexpr int pitch(int t) { return width(t); }
  static constexpr int chunks(int t) { return width(t) / VL; }  // of a row
  template <int t> static __device__ __forceinline__ int swz(int r) {
    if constexpr (chunks(t) % 16 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (chunks(t) % 8 == 0) return ((r & 2) << 1) | ((r >> 2) & 3);
    else return (r >> 2) & 3;
  }
  static constexpr int tile_off(int t) {  // bytes, within one stage
    int o = 0;
    for (int i = 0; i < t; ++i) o += P::TS * pitch(i) * (int)sizeof(T);
    return o;
  }
  static constexpr int tab_off = tile_off(P::NST);
  static constexpr int stage_bytes = tab_off + P::NTAB * P::TS * 4;
  static constexpr int group_bytes = P::STAGES * stage_bytes;
  static constexpr int tiles_bytes = NG * group_bytes;
  static constexpr int nreg() {  // accumulator registers of a lane
    int n = 0;
    for (int o = 0; o < P::NOP; ++o) n += width(P::ost(o)) / 2;
    return n;
  }
  static constexpr int merge_bytes = P::WSPLIT ? P::NW * (nreg() + 2) * 64 * 4 : 0;
  static constexpr int bin_bytes = P::NW * P::NBIN * 64 * 4;
  static constexpr int main_bytes = tiles_bytes > merge_bytes ? tiles_bytes : merge_bytes;
  static constexpr int list_off = main_bytes;
  static constexpr int range_off = list_off + kListCap * 2;             // own ranges: [wave][NOV][2]
  static constexpr int misc_off = range_off + (P::NW * P::NOV * 2 + 8) * 4;
  static constexpr int lut_off = (misc_off + 64 + 15) / 16 * 16;
  static constexpr int bin_off = lut_off + (P::LUT + 3) / 4 * 16;
  static constexpr int bytes = bin_off + bin_bytes;
};

// Values that a rarely taken block of vector code starts from: what depends on
// them cannot be evaluated ahead of the block (the compiler would evaluate all
// of it always and select the results afterwards).
__device__ __forceinline__ float rare(float v) {
  asm volatile("" : "+v"(v));
  return v;
}

// An address in LDS of which the compiler knows no part: small constant offsets
// from it fit the loads (with a known part it adds that per load).
typedef const __attribute__((address_space(3))) float* LdsFloat;
__device__ __forceinline__ LdsFloat lds_base(const float* p) {
  LdsFloat q = (LdsFloat)p;
  asm("" : "+v"(q));
  return q;
}

// tanh with the fp32 accuracy that scores need (absolute: a few 2^-24), as one
// exponential and one reciprocal: 1 - 2 / (e^{2x} + 1).
// pl_ctanh: c tanh(a x) without the products by a and c, for |c| up to 256: the
// absolute error, a few 2^-24 of c, is then below what 16-bit operands give scores.
__device__ __forceinline__ float pl_ctanh(float x, float a, float c) {
  return __builtin_fmaf(-2.0f * c, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (a * 2.0f * kLog2e)) + 1.0f), c);
}
__device__ __forceinline__ float pl_tanh(float x) { return pl_ctanh(x, 1.0f, 1.0f); }
__device__ __forceinline__ float pl_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// exp(x) 2^sx
__device__ __forceinline__ float pl_exp_by(float x, float sx) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, sx)); }

template <int V> struct ic {
  static constexpr int value = V;
};

template <int N, int I = 0, class F> __device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(ic<I>{});
    static_for<N, I + 1>(f);
  }
}

template <int GT> __device__ __forceinline__ void group_sync() {
  if constexpr (GT > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// Minima and maxima over 8 or 16 neighbouring lanes by data-parallel moves
// (within quads, then mirrored halves and rows), over the wave by reading one
// lane of each row, over a lane and its partner 32 further by a lane swap: none
// waits for LDS as the general shuffle does.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}
template <int N> __device__ __forceinline__ float lanes_min(float v) {
  v = k_min(v, dpp<0xB1>(v));
  v = k_min(v, dpp<0x4E>(v));
  v = k_min(v, dpp<0x141>(v));
  if constexpr (N == 16) v = k_min(v, dpp<0x140>(v));
  return v;
}
template <int N> __device__ __forceinline__ float lanes_max(float v) {
  v = k_max(v, dpp<0xB1>(v));
  v = k_max(v, dpp<0x4E>(v));
  v = k_max(v, dpp<0x141>(v));
  if constexpr (N == 16) v = k_max(v, dpp<0x140>(v));
  return v;
}
__device__ __forceinline__ float from_lane(float v, int l) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
}
__device__ __forceinline__ float wave_min(float v) {
  v = lanes_min<16>(v);
  return k_min(k_min(from_lane(v, 0), from_lane(v, 16)), k_min(from_lane(v, 32), from_lane(v, 48)));
}
__device__ __forceinline__ float wave_max(float v) {
  v = lanes_max<16>(v);
  return k_max(k_max(from_lane(v, 0), from_lane(v, 16)), k_max(from_lane(v, 32), from_lane(v, 48)));
}
struct Halves {
  float a, b;  // of the lane in the lower half and of the one in the upper half
};
__device__ __forceinline__ Halves halves(float v) {
  const unsigned i = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
  return {__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
__device__ __forceinline__ float uniform(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// Sum of x y over a row of D elements, by the two lanes that own the row.
template <int D, typename T> __device__ __forceinline__ float row_dot(const T* x, const T* y) {
  constexpr int VL = Mma<T>::VL;
  float s = 0.0f;
#pragma unroll 4
  for (int c = ((threadIdx.x >> 5) & 1) * VL; c < D; c += 2 * VL) {
    const vec_t<VL, T> u = *(const vec_t<VL, T>*)(x + c), v = *(const vec_t<VL, T>*)(y + c);
#pragma unroll
    for (int j = 0; j < VL; ++j) s = __builtin_fmaf(tof(u[j]), tof(v[j]), s);
  }
  const Halves r = halves(s);
  return r.a + r.b;
}

// Interval arithmetic on value ranges (rounding is monotone, so a range of
// rounded operations holds the rounded values).  Values that may be anything,
// NaN included, have NaN for both ends: so do vectors with a NaN or an infinity
// (whose differences may be NaN), and what is computed from them; a comparison
// with such a range may be false and may be true.  (No contraction: a fused
// multiply-add would round otherwise than the primitives.)
struct Range {
  float lo, hi;
};
__device__ __forceinline__ bool finite(float v) { return v - v == 0.0f; }
__device__ __forceinline__ Range r_pt(float v) { return {v, v}; }
__device__ __forceinline__ Range r_all() { return {__builtin_nanf(""), __builtin_nanf("")}; }
__device__ __forceinline__ Range r_if(bool known, Range a) { return known ? a : r_all(); }
__device__ __forceinline__ Range r_sum(float lo, float hi) { return r_if(finite(lo) && finite(hi), {lo, hi}); }
__device__ __forceinline__ Range r_add(Range a, Range b) {
#pragma clang fp contract(off)
  return r_sum(a.lo + b.lo, a.hi + b.hi);
}
__device__ __forceinline__ Range r_sub(Range a, Range b) {
#pragma clang fp contract(off)
  return r_sum(a.lo - b.hi, a.hi - b.lo);
}
__device__ __forceinline__ Range r_neg(Range a) { return {-a.hi, -a.lo}; }
__device__ __forceinline__ bool r_known(Range a) { return a.lo == a.lo; }
__device__ __forceinline__ Range r_max(Range a, Range b) { return r_if(r_known(a) && r_known(b), {k_max(a.lo, b.lo), k_max(a.hi, b.hi)}); }
__device__ __forceinline__ Range r_min(Range a, Range b) { return r_if(r_known(a) && r_known(b), {k_min(a.lo, b.lo), k_min(a.hi, b.hi)}); }
__device__ __forceinline__ Range r_mul(Range a, Range b) {
#pragma clang fp contract(off)
  const float p = a.lo * b.lo, q = a.lo * b.hi, r = a.hi * b.lo, s = a.hi * b.hi;
  return r_if(finite(p) && finite(q) && finite(r) && finite(s), {k_min(k_min(p, q), k_min(r, s)), k_max(k_max(p, q), k_max(r, s))});
}
__device__ __forceinline__ Range r_abs(Range a) {
  const float p = __builtin_fabsf(a.lo), q = __builtin_fabsf(a.hi);
  return r_if(r_known(a), {a.lo <= 0.0f && a.hi >= 0.0f ? 0.0f : k_min(p, q), k_max(p, q)});
}
__device__ __forceinline__ Range r_lt(Range a, Range b) { return {a.hi < b.lo ? 1.0f : 0.0f, a.lo >= b.hi ? 0.0f : 1.0f}; }
__device__ __forceinline__ Range r_le(Range a, Range b) { return {a.hi <= b.lo ? 1.0f : 0.0f, a.lo > b.hi ? 0.0f : 1.0f}; }
__device__ __forceinline__ Range r_eq(Range a, Range b) {
  return {a.lo == a.hi && b.lo == b.hi && a.lo == b.lo ? 1.0f : 0.0f, a.lo > b.hi || b.lo > a.hi ? 0.0f : 1.0f};
}

template <class P> struct Plane {
  typedef typename P::T T;
  typedef Geo<P> G;
  typedef Mma<T> M;
  typedef typename M::Frag Frag;
  static constexpr int VL = M::VL, KU = M::KU;
  typedef vec_t<VL, T> V16;
  static constexpr int NREG = G::nreg();

  static constexpr int vpt(int t) { return (P::TS * (P::sw(t) / VL) + G::GT - 1) / G::GT; }  // staging vectors of a thread
  static constexpr int vtot() {
    int n = 0;
    if (G::DMA) return 1;
    for (int t = 0; t < P::NST; ++t) n += vpt(t);
    return n > 0 ? n : 1;
  }
  static constexpr int vbase(int t) {
    int n = 0;
    for (int i = 0; i < t; ++i) n += vpt(i);
    return n;
  }
  static constexpr int kfrag(int p) { return (P::sw(P::sst(p)) + KU - 1) / KU; }
  static constexpr int fbase(int p) {
    int n = 0;
    for (int i = 0; i < p; ++i) n += kfrag(i);
    return n;
  }
  static constexpr int NF = fbase(P::NSP);
  static constexpr int abase(int o) {  // first 32-wide accumulator tile of output product o
    int n = 0;
    for (int i = 0; i < o; ++i) n += G::width(P::ost(i)) / 32;
    return n;
  }
  static constexpr int NA = abase(P::NOP);
  static constexpr int TABV = (P::NTAB * P::TS + G::GT - 1) / G::GT;

  // P::SCALED (fp16 planes that are an exponential times what does not depend on
  // it, as a gradient's P and dX): fp16 has ever fewer bits for values below
  // 2^-14, which a gradient's are with many keys or a small dO, and no number past
  // 65504.  So each output product's values carry a factor 2^n that its results lose
  // in fp32: the first one's is added to the exponential's exponent (sx), the
  // others' multiply their values once more (by[o]).  The factors are an owned
  // index's own; like a softmax's reference they start where the first values put
  // them and move only when values would pass kScaleMost, to where the largest
  // is at most 2^kScaleAt.  (12 heads of 4000 rows, eleven packed documents, width
  // 64: queries' gradients 27.2 us without, 28.1 with; keys' 32.6 and 34.5.  2x16
  // causal heads of 2048: 50.1 and 53.1, 61 and 67; width 128, capped, 95 and 96,
  // 132 and 140.)
  static constexpr float kScaleMost = 65000.0f;
  static constexpr int kScaleAt = 6, kScaleFirst = 40;

  // A softmax's exponentials in fp16 carry a factor 2^7 (at most 2^15 in all then):
  // weights down to 2^-21 of a row's largest keep all bits of the type.  Without it
  // those below 2^-14 lost them: where one key takes nearly all weight the others'
  // share was off by up to 4 %.
  static constexpr float kLift = is_f16<T>::value ? 7.0f : 0.0f;

  const KArgs& a;
  typename P::B b;
  char* smem;
  int tid, wave, lane, l32, h, gt, gtid;
  i64 own0, own1;  // first owned index of the workgroup, end of its block (or axis)
  float ov[P::NOV > 0 ? P::NOV : 1];
  Frag bf[NF];
  f32x16 acc[NA > 0 ? NA : 1];
  float mref, mtrue, lsum;
  float sx, by[P::NOP > 0 ? P::NOP : 1];
  Range wr[P::NOV > 0 ? P::NOV : 1];  // ranges of the owned vectors over the wave
  V16 st[vtot()];
  float stab[TABV > 0 ? TABV : 1];

  __device__ __forceinline__ Plane(const KArgs& a_, char* s) : a(a_), smem(s) {}

  // This lane's owned index (clamped to the block), and whether it exists.
  __device__ __forceinline__ i64 own_raw() const { return own0 + (P::WSPLIT ? 0 : wave * 32) + l32; }
  __device__ __forceinline__ i64 own() const { return own_raw() < own1 ? own_raw() : own1 - 1; }
  __device__ __forceinline__ bool own_ok() const { return own_raw() < own1; }

  __device__ __forceinline__ char* stage(int s) const { return smem + (P::WSPLIT ? wave * G::group_bytes : 0) + s * G::stage_bytes; }

  // ---- loads of one streamed tile ------------------------------------------------
  // Rows are read through a buffer descriptor of the tile's rows that exist:
  // reads past it return zero (rows past the axis, columns past a tensor's
  // width, rows that the operand's own condition excludes).
  template <int t> __device__ __forceinline__ i32x4 tile_rows(i64 s0) const {
    const int rows = P::NSTR - s0 < P::TS ? (int)(P::NSTR - s0) : P::TS;
    const unsigned long long p = (unsigned long long)P::template srow<t>(a, b, s0);
    // in scalar registers, as the loads in assembly need it
    return i32x4{__builtin_amdgcn_readfirstlane((int)(unsigned)p), __builtin_amdgcn_readfirstlane((int)((p >> 32) & 0xffff)),
                 __builtin_amdgcn_readfirstlane(((rows - 1) * P::srs(t) + P::sw(t)) * (int)sizeof(T)), 0x00020000};
  }
  // Byte offset of chunk c of a tile's row, or one past the rows.
  template <int t> __device__ __forceinline__ unsigned tile_offset(i64 s0, int row, int c, bool in) const {
    if constexpr (P::row_mask(t)) {
      const i64 r = s0 + row;
      in = in && P::template srow_ok<t>(a, b, r < P::NSTR ? r : P::NSTR - 1);
    }
    return in ? (unsigned)(row * P::srs(t) * (int)sizeof(T) + c * 16) : 0x80000000u;
  }
  // DMA: straight into the LDS of stage s, 64
  // consecutive chunks per instruction; a lane fetches the chunk that its place
  // holds.  Its wave waits for the loads before the tile is shared (landed()).
  // Otherwise into registers, and from there to LDS when the tile before has been read.
  __device__ __forceinline__ void fetch(int s, i64 s0) {
    // a wave alone has no barrier between its last reads of the stage and the loads that overwrite it
    if constexpr (G::DMA && G::GT == 64) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    static_for<P::NST>([&](auto ti) {
      constexpr int t = decltype(ti)::value;
      const i32x4 rs = tile_rows<t>(s0);
      if constexpr (G::DMA) {
        constexpr int CH = G::chunks(t), NI = P::TS * CH / 64;
        typedef __attribute__((address_space(3))) char lds_char;
        const unsigned to = (unsigned)(unsigned long long)(lds_char*)(stage(s) + G::tile_off(t));
        constexpr int NWG = G::GT / 64;  // waves that share the tile
        const int me = NWG > 1 ? wave : 0;
#pragma unroll
        for (int i = 0; i < NI; i += NWG) {
          if (NI % NWG == 0 || i + me < NI) {
            const int u = (i + me) * 64 + lane, row = u / CH, c = (u % CH) ^ G::template swz<t>(row);
            const unsigned off = tile_offset<t>(s0, row, c, c < P::sw(t) / VL);
            const unsigned la = __builtin_amdgcn_readfirstlane(to + (i + me) * 1024);
            // (the descriptor may come straight from vector instructions: five wait states)
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" ::"v"(off), "s"(la), "s"(rs) : "memory", "m0");
          }
        }
      } else {
        constexpr int CV = P::sw(t) / VL;
        const __amdgpu_buffer_rsrc_t rr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(P::template srow<t>(a, b, s0)), 0, rs[2], 0x00020000);
#pragma unroll
        for (int i = 0; i < vpt(t); ++i) {
          const int e = gtid + i * G::GT, row = e / CV, c = e % CV;
          const bool in = (P::TS * CV) % G::GT == 0 || e < P::TS * CV;
          st[vbase(t) + i] = __builtin_bit_cast(V16, __builtin_amdgcn_raw_buffer_load_b128(rr, tile_offset<t>(s0, row, c, in), 0, 0));
        }
      }
    });
    if constexpr (P::NTAB > 0) {
#pragma unroll
      for (int i = 0; i < TABV; ++i) {
        const int e = gtid + i * G::GT;
        const int k = e / P::TS;
        const i64 r = s0 + e % P::TS, rc = r < P::NSTR ? r : P::NSTR - 1;
        stab[i] = k < P::NTAB ? P::tab(a, b, k, rc) : 0.0f;
      }
    }
  }
  __device__ __forceinline__ void put(int s) {
    char* base = stage(s);
    if constexpr (!G::DMA)
      static_for<P::NST>([&](auto ti) {
        constexpr int t = decltype(ti)::value;
        constexpr int CV = P::sw(t) / VL;
#pragma unroll
        for (int i = 0; i < vpt(t); ++i) {
          const int e = gtid + i * G::GT, row = e / CV, c = e % CV;
          if ((P::TS * CV) % G::GT == 0 || e < P::TS * CV)
            *(V16*)((T*)(base + G::tile_off(t)) + row * G::pitch(t) + (c ^ G::template swz<t>(row)) * VL) = st[vbase(t) + i];
        }
      });
    if constexpr (P::NTAB > 0) {
#pragma unroll
      for (int i = 0; i < TABV; ++i) {
        const int e = gtid + i * G::GT;
        if (e < P::NTAB * P::TS) ((float*)(base + G::tab_off))[e] = stab[i];
      }
    }
  }
  // This wave's loads have arrived, the direct ones included.  As a builtin, so
  // that the compiler knows it of its own loads: the owned operands' are done
  // before the walk.  (Else it waits for them in every tile, with vmcnt(0), and
  // so for the next tile's direct loads, which it cannot count.)
  static __device__ __forceinline__ void landed() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    asm volatile("" ::: "memory");
  }
  // Columns past a tensor's width take part in the score products: zeros
  // (direct loads write them with every tile).
  __device__ __forceinline__ void clear_pads() {
    if constexpr (!G::DMA)
      static_for<P::NST>([&](auto ti) {
        constexpr int t = decltype(ti)::value;
        constexpr int PV = (G::width(t) - P::sw(t)) / VL;
        if constexpr (PV > 0)
          for (int s = 0; s < P::STAGES; ++s)
            for (int e = gtid; e < P::TS * PV; e += G::GT)
              *(V16*)((T*)(stage(s) + G::tile_off(t)) + (e / PV) * G::pitch(t) + ((P::sw(t) / VL + e % PV) ^ G::template swz<t>(e / PV)) * VL) = V16{};
      });
  }

  // ---- products --------------------------------------------------------------
  template <int p> __device__ __forceinline__ f32x16 score(const char* base, int sub) const {
    constexpr int t = P::sst(p);
    f32x16 c = {};
    const T* q = (const T*)(base + G::tile_off(t)) + (sub * 32 + l32) * G::pitch(t);
    const int z = h ^ G::template swz<t>(l32);
    if constexpr (G::DMA && kfrag(p) <= 8) {
      // all reads go out before the first product waits for one (2x16 causal capped
      // heads of 2048, width 128: 69.5 -> 67.2 us, gradients 99 -> 97 and 145 -> 141);
      // a tile in registers or wider operands leave no registers for that
      Frag f[kfrag(p)];
#pragma unroll
      for (int k = 0; k < kfrag(p); ++k) f[k] = *(const Frag*)(q + ((2 * k) ^ z) * VL);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < kfrag(p); ++k) c = M::run(f[k], bf[fbase(p) + k], c);
    } else {
#pragma unroll
      for (int k = 0; k < kfrag(p); ++k) c = M::run(*(const Frag*)(q + ((2 * k) ^ z) * VL), bf[fbase(p) + k], c);
    }
    return c;
  }
  template <int o> __device__ __forceinline__ void output(const char* base, int sub, const float* X) {
    constexpr int t = P::ost(o);
    constexpr int ND = G::width(t) / 32;
    const T* w = (const T*)(base + G::tile_off(t));
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        // The plane's values are rounded to the operands' type: the matrix
        // instructions take nothing else, two parts of a value would double this
        // product, and in its sums such errors average out like the result's own
        // rounding.  Statistics and sums keep the unrounded values.
        Frag x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fromf<T>(P::SCALED && o > 0 ? X[8 * kk + j] * by[o] : X[8 * kk + j]);
        // this lane's part of a read: row r (and r + 8), columns 8 c + 4 (lane & 1) .. + 3 of 32
        const int r = 4 * h + ((lane & 15) >> 2), c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        const T* r0 = w + (sub * 32 + kk * 16 + r) * G::pitch(t) + 4 * (lane & 1);
        const int z0 = c ^ G::template swz<t>(r), z1 = c ^ G::template swz<t>(r + 8);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(r0 + ((4 * d) ^ z0) * VL));
          s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(r0 + 8 * G::pitch(t) + ((4 * d) ^ z1) * VL));
          acc[abase(o) + d] = M::run(__builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), x, acc[abase(o) + d]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i / 4) + 4 * h + i % 4;
        const T* r0 = w + (sub * 32 + r) * G::pitch(t) + l32 % 4;
        const int z = (l32 / 4) ^ G::template swz<t>(r);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          acc[abase(o) + d] = __builtin_amdgcn_mfma_f32_32x32x2f32(r0[((8 * d) ^ z) * VL], X[i], acc[abase(o) + d], 0, 0, 0);
      }
    }
  }

  // With one wave per SIMD accumulators live in accumulation registers, which
  // vector instructions do not reach.  A block that is rarely taken and multiplies
  // them fetches and returns them itself with this at its ends (else they are
  // copied with every subtile: keys' gradients of 2x16 causal heads of 2048, width
  // 128, fp16, 15 us more).
  __device__ __forceinline__ void home() {
    if constexpr (P::WPE == 1)
#pragma unroll
      for (int d = 0; d < NA; ++d) asm volatile("" : "+a"(acc[d]));
  }
  // 2^-sx
  __device__ __forceinline__ float unscaled() const { return __builtin_ldexpf(1.0f, -(int)sx); }
  // Moves the scales where values of this subtile outgrow them.
  __device__ __forceinline__ void rescale(float (*X)[16]) {
    float top[P::NOP > 0 ? P::NOP : 1];
    bool past = false;
    static_for<P::NOP>([&](auto oi) {
      constexpr int o = decltype(oi)::value, k = P::ox(o);
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) t = k_max(t, __builtin_fabsf(X[k][i]));
      const Halves th = halves(t);
      top[o] = o ? k_max(th.a, th.b) * by[o] : k_max(th.a, th.b);
      past = past || top[o] > kScaleMost;
    });
    if (__any(past)) {
      home();
      static_for<P::NOP>([&](auto oi) {
        constexpr int o = decltype(oi)::value;
        // (an infinity stays one whatever the scale)
        const float t = rare(top[o]);
        const int e = t > (float)(1 << kScaleAt) && finite(t) ? kScaleAt - __builtin_amdgcn_frexp_expf(t) : 0;
        const float f = __builtin_ldexpf(1.0f, e);
        if constexpr (o == 0) {
          sx += (float)e;
          for (int q = 1; q < P::NOP; ++q) by[q] *= __builtin_ldexpf(1.0f, -e);
#pragma unroll
          for (int k = 0; k < P::NX; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) X[k][i] *= f;
        } else {
          by[o] *= f;
        }
#pragma unroll
        for (int d = abase(o); d < abase(o + 1); ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= f;
      });
      home();
    }
  }

  // Streamed index (within its tile) of register i of subtile sub.
  __device__ __forceinline__ int sidx(int sub, int i) const { return sub * 32 + 8 * (i / 4) + 4 * h + i % 4; }

  // f(i, values of the streamed vectors, bases of the looked-up tables and offset
  // from them, streamed index (clamped), it exists) for the registers of a subtile.
  template <class F> __device__ __forceinline__ void elements(const char* base, i64 s0, int sub, F&& f) {
    const float* tab = (const float*)(base + G::tab_off);
    const int rows = P::NSTR - s0 < P::TS ? (int)(P::NSTR - s0) : P::TS;
    LdsFloat lb[P::NLUT > 0 ? P::NLUT : 1];
    P::bases(ov, (const float*)(smem + G::lut_off), s0 + sub * 32 + 4 * h, lb);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 tv4[P::NTAB > 0 ? P::NTAB : 1];
#pragma unroll
      for (int k = 0; k < P::NTAB; ++k) tv4[k] = *(const f32x4*)(tab + k * P::TS + sub * 32 + 8 * g + 4 * h);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float tv[P::NTAB > 0 ? P::NTAB : 1];
#pragma unroll
        for (int k = 0; k < P::NTAB; ++k) tv[k] = tv4[k][r];
        const int s = sidx(sub, 4 * g + r);
        f(4 * g + r, tv, lb, 8 * g + r, s0 + (s < rows ? s : rows - 1), s < rows);
      }
    }
  }

  // ---- one tile ---------------------------------------------------------------
  // `full`: no pair of the tile is masked and every streamed index exists.  The
  // mask is a step of its own, so that both kinds of tiles share the products.
  __device__ __forceinline__ void tile(int s, i64 s0, bool full) {
    const char* base = stage(s);
    const float* lut = (const float*)(smem + G::lut_off);
    if constexpr (P::SOFTMAX) {
      f32x16 x[G::NSUB];
#pragma unroll
      for (int sub = 0; sub < G::NSUB; ++sub) x[sub] = score<0>(base, sub);
#pragma unroll
      for (int sub = 0; sub < G::NSUB; ++sub)
        elements(base, s0, sub, [&](int i, const float* tv, const LdsFloat* lb, int kk, i64 sc, bool) {
          float xs[1] = {x[sub][i]};
          x[sub][i] = P::logit(a, b, ov, tv, lut, lb, kk, own(), sc, xs);
        });
      if (!full) {
        float om[P::NOV > 0 ? P::NOV : 1];
        for (int k = 0; k < P::NOV; ++k) om[k] = rare(ov[k]);
        const float minus = rare(-__builtin_huge_valf());
        // a masked pair's score is -inf: its exponential is 0 whatever the maximum
#pragma unroll
        for (int sub = 0; sub < G::NSUB; ++sub)
          elements(base, s0, sub, [&](int i, const float* tv, const LdsFloat* lb, int kk, i64 sc, bool ok) {
            x[sub][i] = ok && P::keep(a, b, om, tv, lut, lb, kk, own(), sc) ? x[sub][i] : minus;
          });
      }
      float top = x[0][0];
#pragma unroll
      for (int sub = 0; sub < G::NSUB; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = k_max(top, x[sub][i]);
      const Halves th = halves(top);
      top = k_max(th.a, th.b);
      mtrue = k_max(mtrue, top);
      if (__any(mtrue > mref + kLazy / P::FOLD)) {
        const float f = rare(mref) == mtrue ? 1.0f : __builtin_amdgcn_exp2f((mref - mtrue) * (P::FOLD * kLog2e));
        mref = mtrue;
        lsum *= f;
#pragma unroll
        for (int d = 0; d < NA; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= f;
      }
      const float mz = mref == -__builtin_huge_valf() ? 0.0f : mref;
      const float mc = kLift - mz * (P::FOLD * kLog2e);
#pragma unroll
      for (int sub = 0; sub < G::NSUB; ++sub) {
        float X[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if constexpr (sizeof(T) == 2)
            X[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[sub][i], P::FOLD * kLog2e, mc));
          else
            X[i] = expf((x[sub][i] - mz) * P::FOLD);
          lsum += X[i];
        }
        static_for<P::NOP>([&](auto oi) { output<decltype(oi)::value>(base, sub, X); });
      }
    } else {
#pragma unroll 1
      for (int sub = 0; sub < G::NSUB; ++sub) {
        f32x16 x[P::NSP];
        static_for<P::NSP>([&](auto pi) { x[decltype(pi)::value] = score<decltype(pi)::value>(base, sub); });
        float X[P::NX][16];
        elements(base, s0, sub, [&](int i, const float* tv, const LdsFloat* lb, int kk, i64 sc, bool) {
          float xs[P::NSP], out[P::NX];
#pragma unroll
          for (int p = 0; p < P::NSP; ++p) xs[p] = x[p][i];
          P::plane(a, b, ov, tv, lut, lb, kk, own(), sc, xs, sx, out);
#pragma unroll
          for (int k = 0; k < P::NX; ++k) X[k][i] = out[k];
        });
        if (!full) {
          float om[P::NOV > 0 ? P::NOV : 1];
          for (int k = 0; k < P::NOV; ++k) om[k] = rare(ov[k]);
          const float zero = rare(0.0f);
          elements(base, s0, sub, [&](int i, const float* tv, const LdsFloat* lb, int kk, i64 sc, bool ok) {
            const bool k1 = ok && P::keep(a, b, om, tv, lut, lb, kk, own(), sc);
#pragma unroll
            for (int k = 0; k < P::NX; ++k) X[k][i] = k1 ? X[k][i] : zero;
          });
        }
        if constexpr (P::SCALED) rescale(X);
        static_for<P::NOP>([&](auto oi) { output<decltype(oi)::value>(base, sub, X[P::ox(decltype(oi)::value)]); });
        if constexpr (P::NBIN > 0) bins(base, s0, sub, X[P::XBIN]);
      }
    }
  }

  // ---- sums of plane values by bin -----------------------------------------------
  // Every lane adds its values to bins of its own in LDS ([bin][lane]): no two
  // lanes meet at an address and a lane's additions keep their order, so the
  // sums do not depend on timing.  The lanes are summed at the end.  Four values
  // are added at a time (their old sums are read together; values that share a
  // bin add up first, and all of them write the same sum), so a subtile waits
  // for LDS four times, not sixteen (8 x 12 heads of 512 x 512, width 64, 32 bins:
  // 39.6 us; values one at a time took 11 us more, LDS atomic additions 146).  Where the index lies past one end of its
  // table for every pair, as far from the diagonal, there is one bin.
  __device__ __forceinline__ void bins(const char* base, i64 s0, int sub, const float* X) {
    float* mine = (float*)(smem + G::bin_off) + wave * (P::NBIN * 64) + lane;
    const float* lut = (const float*)(smem + G::lut_off);
    const Range e = P::bin_range(a, b, wr, (float)(s0 + sub * 32), (float)(s0 + sub * 32 + 31));
    const bool live = own_ok();
    const float back = P::SCALED ? unscaled() : 1.0f;
    if (e.lo >= (float)(P::BIN_T - 1) || e.hi <= 0.0f) {
      const int k = (int)P::bin_end(lut, e.hi > 0.0f);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += X[i];  // zero past the axis
      mine[k * 64] += live ? sum * back : 0.0f;
      return;
    }
    int id[16];
    elements(base, s0, sub, [&](int i, const float* tv, const LdsFloat* lb, int kk, i64 sc, bool) { id[i] = (int)P::bin(a, b, ov, tv, lut, lb, kk, own(), sc) * 64; });
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float old[4], add[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) old[i] = mine[id[4 * g + i]];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        add[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) add[i] += id[4 * g + j] == id[4 * g + i] ? X[4 * g + j] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[id[4 * g + i]] = old[i] + (live ? add[i] * back : 0.0f);
    }
  }

  // ---- the kernel --------------------------------------------------------------
  __device__ __forceinline__ void run() {
    tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;
    gtid = P::WSPLIT ? lane : tid;
    // Order of the work.  An owned axis is made of blocks of SEG indices and TP
    // tiles (the positions of one head) along which a mask usually changes the work
    // steadily.  The longest tiles of all blocks come first; of the workgroups
    // that are resident from the start (OCC per compute unit) every second round
    // over the compute units runs backwards, so that a long and a short one
    // share a compute unit.  Workgroups are dealt to
    // the eight XCDs in turn: with whole blocks for each, a block's streamed rows
    // stay in one XCD's L2.
    constexpr int NBLK = P::NB * (P::OTILES / P::TP);
    constexpr bool by_xcd = NBLK % 8 == 0;
    constexpr int NX = by_xcd ? NBLK / 8 : NBLK, CHUNK = by_xcd ? 32 : 256, ITEMS = NX * P::TP * P::SPLIT;
    const int x0 = by_xcd ? (blockIdx.x & 7) * NX : 0;
    int w = by_xcd ? blockIdx.x >> 3 : blockIdx.x;
    const int round = w / CHUNK;
    if (round < P::OCC && (round & 1)) w = round * CHUNK + (ITEMS - round * CHUNK < CHUNK ? ITEMS - round * CHUNK : CHUNK) - 1 - w % CHUNK;
    const int z = w % P::SPLIT, blk = x0 + w / P::SPLIT % NX, rank = w / P::SPLIT / NX;
    const int bl = blk / (P::OTILES / P::TP), ot = blk % (P::OTILES / P::TP) * P::TP + (P::LAST_FIRST ? P::TP - 1 - rank : rank);
    b = P::batch(bl);
    own0 = (i64)(ot / P::TP) * P::SEG + (i64)(ot % P::TP) * G::OT;
    own1 = (i64)(ot / P::TP + 1) * P::SEG;
#pragma unroll
    for (int k = 0; k < P::NOV; ++k) ov[k] = P::own(a, b, k, own());
    // owned fragments
    static_for<P::NSP>([&](auto pi) {
      constexpr int p = decltype(pi)::value;
      const T* r = P::template orow<p>(a, b, own());
      bool ok = own_ok();
      if constexpr (P::own_mask(p)) ok = ok && P::template orow_ok<p>(a, b, own());
#pragma unroll
      for (int k = 0; k < kfrag(p); ++k) {
        const int c = k * KU + h * (KU / 2);
        Frag v = {};
        if (ok && c < P::sw(P::sst(p))) v = *(const Frag*)(r + c);
        bf[fbase(p) + k] = v;
      }
    });
#pragma unroll
    for (int d = 0; d < NA; ++d) acc[d] = f32x16{};
    mref = mtrue = P::MINIT;
    lsum = 0.0f;
    sx = (float)kScaleFirst;
#pragma unroll
    for (int o = 0; o < P::NOP; ++o) by[o] = 1.0f;
    if constexpr (P::NBIN > 0)
      for (int k = 0; k < P::NBIN; ++k) ((float*)(smem + G::bin_off))[(wave * P::NBIN + k) * 64 + lane] = 0.0f;
    clear_pads();
    // tables that the plane looks up, as the values it reads
    if constexpr (P::LUT > 0) {
      for (int k = tid; k < P::LUT; k += G::NT) ((float*)(smem + G::lut_off))[k] = P::lut_value(a, b, k);
      __syncthreads();
    }
    // ranges of the owned vectors, over the workgroup and over the wave
    float* rng = (float*)(smem + G::range_off);
    Range gr[P::NOV > 0 ? P::NOV : 1];
    // (only of those that the mask or the bins compare: the others are still on their way)
    if constexpr (P::MASK || P::NBIN > 0) {
      static_for<P::NOV>([&](auto ki) {
        constexpr int k = decltype(ki)::value;
        if constexpr (P::ranged(k)) {
          const bool bad = __any(!finite(ov[k]));
          wr[k] = bad ? r_all() : Range{uniform(wave_min(ov[k])), uniform(wave_max(ov[k]))};
          if (lane == 0) rng[(wave * P::NOV + k) * 2] = wr[k].lo, rng[(wave * P::NOV + k) * 2 + 1] = wr[k].hi;
        }
      });
      __syncthreads();
      static_for<P::NOV>([&](auto ki) {
        constexpr int k = decltype(ki)::value;
        if constexpr (P::ranged(k)) {
          gr[k] = wr[k];
          for (int v = 0; v < P::NW; ++v) {
            const Range o = {rng[(v * P::NOV + k) * 2], rng[(v * P::NOV + k) * 2 + 1]};
            gr[k] = r_if(r_known(gr[k]) && r_known(o), {k_min(gr[k].lo, o.lo), k_max(gr[k].hi, o.hi)});
          }
        }
      });
    }
    unsigned short* list = (unsigned short*)(smem + G::list_off);
    int* misc = (int*)(smem + G::misc_off);
    constexpr int ntiles = (int)((P::NSTR + P::TS - 1) / P::TS);
    for (int c0 = 0; c0 < ntiles; c0 += kListCap) {
      const int cn = ntiles - c0 < kListCap ? ntiles - c0 : kListCap;
      int n = cn;
      if constexpr (P::MASK) {
        __syncthreads();  // the previous chunk's list is no longer read
        // state of each tile: 0 no pair, 1 some, 2 all; a group of TS / 4 lanes
        // reads the tile's vectors
        constexpr int GL = P::TS / 4, TPI = P::NRV ? G::NT / GL : G::NT;  // tiles of one step
        constexpr int U = P::NRV ? 4 : 1;                                 // steps whose loads go out together
        for (int t0 = 0; t0 < cn; t0 += U * TPI) {
          float val[U][P::NRV > 0 ? P::NRV : 1][4];
          auto first = [&](int u) {
            const int t = t0 + u * TPI + (P::NRV ? tid / GL : tid);
            return (i64)(c0 + (t < cn ? t : cn - 1)) * P::TS;
          };
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < P::NRV; ++k)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const i64 r = first(u) + (tid % GL) * 4 + j;
                val[u][k][j] = P::rvec(a, b, k, r < P::NSTR ? r : P::NSTR - 1);
              }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int t = t0 + u * TPI + (P::NRV ? tid / GL : tid);
            const i64 s0 = first(u);
            Range rv[P::NRV > 0 ? P::NRV : 1];
#pragma unroll
            for (int k = 0; k < P::NRV; ++k) {
              float lo = __builtin_huge_valf(), hi = -lo;
              bool bad = false;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float v = val[u][k][j];
                bad = bad || !finite(v);
                lo = k_min(lo, v), hi = k_max(hi, v);
              }
              // (an infinite end of the group marks it)
              if (bad) lo = -__builtin_huge_valf(), hi = -lo;
              rv[k] = r_sum(lanes_min<GL>(lo), lanes_max<GL>(hi));
            }
            const i64 s1 = s0 + P::TS - 1 < P::NSTR - 1 ? s0 + P::TS - 1 : P::NSTR - 1;
            const Range c = P::mask_range(a, b, gr, rv, (float)s0, (float)s1);
            // (a select takes every value that is not 0 as true, negative ones too)
            const int state = c.lo == 0.0f && c.hi == 0.0f ? 0 : ((c.lo > 0.0f || c.hi < 0.0f) && s0 + P::TS <= P::NSTR ? 2 : 1);
            if (t < cn && (!P::NRV || tid % GL == 0)) list[t] = (unsigned short)state;
          }
        }
        __syncthreads();
        // compaction by one wave, in order (entries move towards the front)
        if (wave == 0) {
          int m = 0;
          for (int t0 = 0; t0 < cn; t0 += 64) {
            const int state = t0 + lane < cn ? list[t0 + lane] : 0;
            const unsigned long long act = __ballot(state != 0);
            const int at = m + __popcll(act & ((1ull << lane) - 1ull));
            if (state) list[at] = (unsigned short)((t0 + lane) | (state == 2 ? 0x8000 : 0));
            m += __popcll(act);
          }
          if (lane == 0) misc[0] = m;
        }
        __syncthreads();
        n = misc[0];
      }
      auto entry = [&](int e, i64& s0, bool& full) {
        if constexpr (P::MASK) {
          const int v = __builtin_amdgcn_readfirstlane((int)list[e]);
          s0 = (i64)(c0 + (v & 0x7fff)) * P::TS;
          full = (v & 0x8000) != 0;
        } else {
          s0 = (i64)(c0 + e) * P::TS;
          full = s0 + P::TS <= P::NSTR;
        }
      };
      // entries e = first, first + step, ...: over the splits and, when the
      // waves split the streamed axis, over the waves
      const int step = P::SPLIT * G::NG, first = z * G::NG + (P::WSPLIT ? wave : 0);
      i64 s0 = 0, sn = 0;
      bool full = false, fulln = false;
      int e = __builtin_amdgcn_readfirstlane(first);
      if (c0 > 0) group_sync<G::GT>();
      if (e < n) {
        entry(e, s0, full);
        fetch(0, s0);
        put(0);
      }
      landed();
      group_sync<G::GT>();
      int s = 0;
      for (; e < n; e += step) {
        const bool more = e + step < n;
        // a stage of its own, or registers: the next tile's loads go out before this tile's work
        constexpr bool ahead = P::STAGES == 2 || !G::DMA;
        if (more) {
          entry(e + step, sn, fulln);
          if constexpr (ahead) fetch(s ^ 1, sn);
        }
        tile(s, s0, full);
        if constexpr (P::STAGES == 1) group_sync<G::GT>();
        if (more) {
          if constexpr (!ahead) fetch(0, sn);
          put(P::STAGES == 1 ? 0 : s ^ 1);
          if constexpr (G::DMA) landed();
        }
        group_sync<G::GT>();
        if constexpr (P::STAGES == 2) s ^= 1;
        s0 = sn, full = fulln;
      }
    }
    finish(bl, ot, z);
  }

  // ---- joining the waves and the splits, and the results -------------------------
  // The row's maximum as the graph defines it (rows without a pair: the mask's own value).
  __device__ __forceinline__ float top_score() const { return mtrue == P::MINIT ? P::LOW : mtrue * P::FOLD; }
  __device__ __forceinline__ void store_group(int at, f32x4 v) {  // register group `at` (4 registers) of the lane
    static_for<P::NOP>([&](auto oi) {
      constexpr int o = decltype(oi)::value;
      constexpr int lo = abase(o) * 4, hi = abase(o + 1) * 4;
      if (at >= lo && at < hi) {
        const int dim = ((at - lo) / 4) * 32 + 8 * ((at - lo) % 4) + 4 * h;
        if (own_ok() && dim < P::sw(P::ost(o))) P::template store<o>(a, b, own(), dim, top_score(), lsum, v);
      }
    });
  }

  __device__ __forceinline__ void finish(int bl, int ot, int z) {
    constexpr int NGRP = NREG / 4;
    if constexpr (P::ROWOUT)
      if (own_ok() && h == 0 && z == 0 && (!P::WSPLIT || wave == 0)) P::row_out(a, b, own(), ov);
    if constexpr (P::NBIN > 0) join_bins(bl, ot, z);
    if constexpr (P::SCALED) {
      const float back = unscaled();
      static_for<P::NOP>([&](auto oi) {
        constexpr int o = decltype(oi)::value;
        const float f = o ? back / by[o] : back;
#pragma unroll
        for (int d = abase(o); d < abase(o + 1); ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= f;
      });
    }
    if constexpr (P::SOFTMAX) {
      const Halves lh = halves(lsum);
      lsum = lh.a + lh.b;
      // to the true maximum
      const float f = __builtin_amdgcn_exp2f((mref == mtrue ? 0.0f : (mref - mtrue) * (P::FOLD * kLog2e)) - kLift);
      lsum *= f;
#pragma unroll
      for (int d = 0; d < NA; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= f;
    }
    if constexpr (P::NOP == 0) {
      // bins only: join_bins has joined the waves and the splits
    } else if constexpr (!P::WSPLIT && P::SPLIT == 1) {
#pragma unroll
      for (int g = 0; g < NGRP; ++g) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = acc[g / 4][(g % 4) * 4 + r];
        store_group(g, v);
      }
      if constexpr (P::SOFTMAX)
        if (own_ok() && h == 0) P::stats(a, b, own(), top_score(), lsum);
    } else {
      constexpr int NM = NGRP + 1;  // groups of four registers, then (m, l)
      float* lds = (float*)smem;
      f32x4 v[NGRP > 0 ? NGRP : 1];
      constexpr int share = P::WSPLIT ? (NGRP + P::NW - 1) / P::NW : NGRP;
      const int g0 = P::WSPLIT ? wave * share : 0;
      if constexpr (P::WSPLIT) {
        __syncthreads();  // the tiles are no longer read
#pragma unroll
        for (int g = 0; g < NGRP; ++g) {
          f32x4 x;
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] = acc[g / 4][(g % 4) * 4 + r];
          *(f32x4*)(lds + ((wave * NGRP + g) * 64 + lane) * 4) = x;
        }
        float* ml = lds + P::NW * NGRP * 256;
        if constexpr (P::SOFTMAX) ml[(wave * 2) * 64 + lane] = mtrue, ml[(wave * 2 + 1) * 64 + lane] = lsum;
        __syncthreads();
        float f[P::NW];
        if constexpr (P::SOFTMAX) {
          float m = P::MINIT, l = 0.0f;
#pragma unroll
          for (int v2 = 0; v2 < P::NW; ++v2) m = k_max(m, ml[v2 * 128 + lane]);
#pragma unroll
          for (int v2 = 0; v2 < P::NW; ++v2) {
            const float mv = ml[v2 * 128 + lane];
            f[v2] = mv == m ? 1.0f : __builtin_amdgcn_exp2f((mv - m) * (P::FOLD * kLog2e));
            l += ml[v2 * 128 + 64 + lane] * f[v2];
          }
          mtrue = m, lsum = l;
        }
#pragma unroll
        for (int g = 0; g < share; ++g) {
          f32x4 s = {};
          if (g0 + g < NGRP)
#pragma unroll
            for (int v2 = 0; v2 < P::NW; ++v2) {
              const f32x4 x = *(const f32x4*)(lds + ((v2 * NGRP + g0 + g) * 64 + lane) * 4);
              if constexpr (P::SOFTMAX) s += x * f[v2];
              else s += x;
            }
          v[g] = s;
        }
      } else {
#pragma unroll
        for (int g = 0; g < NGRP; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) v[g][r] = acc[g / 4][(g % 4) * 4 + r];
      }
      if constexpr (P::SPLIT > 1) {
        // partial results, [batch and owned tile][split][wave][group][lane]
        constexpr int WV = P::WSPLIT ? 1 : P::NW;
        const int wv = P::WSPLIT ? 0 : wave;
        const i64 cell = (i64)bl * P::OTILES + ot;
        float* part = (float*)a.p[P::SCR] + cell * ((i64)P::SPLIT * WV * NM * 256);
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(part, 0, (int)(P::SPLIT * WV * NM * 1024), 0x00020000);
        auto at = [&](int zz, int g) { return (unsigned)((((zz * WV + wv) * NM + g) * 64 + lane) * 16); };
#pragma unroll
        for (int g = 0; g < share; ++g)
          if (g0 + g < NGRP) coherent_store4(rs, at(z, g0 + g), float4{v[g][0], v[g][1], v[g][2], v[g][3]});
        if constexpr (P::SOFTMAX)
          if (!P::WSPLIT || wave == 0) coherent_store4(rs, at(z, NGRP), float4{mtrue, lsum, 0.0f, 0.0f});
        __builtin_amdgcn_s_waitcnt(0);  // this wave's partial stores are performed
        __syncthreads();
        int* misc = (int*)(smem + G::misc_off);
        if (tid == 0) {
          int* cnt = (int*)a.p[P::CNT] + cell * 32;
          const int old = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          misc[1] = old == P::SPLIT - 1;
          if (old == P::SPLIT - 1) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!misc[1]) return;
        auto factor = [&](float mv) { return mv == mtrue ? 1.0f : __builtin_amdgcn_exp2f((mv - mtrue) * (P::FOLD * kLog2e)); };
        // Rounds of up to 32 vectors of partial results: a round trip to the
        // device's point of coherence is 1 to 2 us.  Unrolled, the compiler puts the
        // loads of several rounds in flight (keys' gradients of 300 rows, 4 heads on
        // 1, width 64, bf16: 8.6 us, 9.6 one round at a time), but past these vectors
        // it spills them (width 224: 23 us, 15.5; one token, 4 fp32 heads of width
        // 208 in 16 splits: 1140 registers, 133 us and 32).
        constexpr int ZB = share >= 32 ? 1 : P::SPLIT < 32 / share ? P::SPLIT : 32 / share;
        constexpr bool flat = P::SPLIT * share <= (P::WPE == 1 ? 112 : 48);
        float ls[P::SPLIT], f[P::SPLIT];
        if constexpr (P::SOFTMAX) {
          mtrue = P::MINIT, lsum = 0.0f;
#pragma unroll
          for (int zz = 0; zz < P::SPLIT; ++zz) {
            const float4 q = coherent_load4(rs, at(zz, NGRP));
            f[zz] = q.x, ls[zz] = q.y;
          }
#pragma unroll
          for (int zz = 0; zz < P::SPLIT; ++zz) mtrue = k_max(mtrue, f[zz]);
          if constexpr (flat)
#pragma unroll
            for (int zz = 0; zz < P::SPLIT; ++zz) {
              f[zz] = factor(f[zz]);
              lsum += ls[zz] * f[zz];
            }
        }
#pragma unroll
        for (int g = 0; g < share; ++g) v[g] = f32x4{};
        auto round = [&](int z0) {
          float4 q[ZB][share], mq[ZB];
#pragma unroll
          for (int zz = 0; zz < ZB; ++zz) {
            const int zc = z0 + zz < P::SPLIT ? z0 + zz : P::SPLIT - 1;
            if constexpr (P::SOFTMAX && !flat) mq[zz] = coherent_load4(rs, at(zc, NGRP));
#pragma unroll
            for (int g = 0; g < share; ++g) q[zz][g] = coherent_load4(rs, at(zc, g0 + g < NGRP ? g0 + g : NGRP - 1));
          }
#pragma unroll
          for (int zz = 0; zz < ZB; ++zz) {
            if (z0 + zz >= P::SPLIT) continue;
            float fz = 1.0f;
            if constexpr (P::SOFTMAX && flat) fz = f[z0 + zz];
            if constexpr (P::SOFTMAX && !flat) {
              fz = factor(mq[zz].x);
              lsum += mq[zz].y * fz;
            }
#pragma unroll
            for (int g = 0; g < share; ++g) {
              const f32x4 x = {q[zz][g].x, q[zz][g].y, q[zz][g].z, q[zz][g].w};
              if constexpr (P::SOFTMAX) v[g] += x * fz;
              else v[g] += x;
            }
          }
        };
        if constexpr (flat) {
#pragma unroll
          for (int z0 = 0; z0 < P::SPLIT; z0 += ZB) round(z0);
        } else {
#pragma unroll 1
          for (int z0 = 0; z0 < P::SPLIT; z0 += ZB) round(z0);
        }
      }
#pragma unroll
      for (int g = 0; g < share; ++g)
        if (g0 + g < NGRP) store_group(g0 + g, v[g]);
      if constexpr (P::SOFTMAX)
        if (own_ok() && h == 0 && (!P::WSPLIT || wave == 0)) P::stats(a, b, own(), top_score(), lsum);
    }
  }

  // Bins of all workgroups of one table row: partial sums in a fixed order.
  __device__ __forceinline__ void join_bins(int bl, int ot, int z) {
    const int row = P::bin_row(b), member = (P::bin_member(b) * P::OTILES + ot) * P::SPLIT + z;
    constexpr int members = P::BIN_MEMBERS * P::OTILES * P::SPLIT;
    float* part = (float*)a.p[P::BSCR] + (i64)row * members * P::NBIN;
    const float* all = (const float*)(smem + G::bin_off);
    __syncthreads();
    // a wave per bin: the lanes' sums of every wave, then over the lanes
#pragma unroll 4
    for (int k = wave; k < P::NBIN; k += P::NW) {
      float s = 0.0f;
      for (int v = 0; v < P::NW; ++v) s += all[(v * P::NBIN + k) * 64 + lane];
      s = group_sum<64>(s);
      if (lane == 0) coherent_store(&part[(i64)member * P::NBIN + k], s);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    int* misc = (int*)(smem + G::misc_off);
    if (tid == 0) {
      int* cnt = (int*)a.p[P::BCNT] + row * 32;
      const int old = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      misc[2] = old == members - 1;
      if (old == members - 1) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!misc[2]) return;
    float* red = (float*)smem;  // [groups][NBIN]
    constexpr int NG2 = P::NBIN < G::NT ? G::NT / P::NBIN : 1;
    for (int k = tid % (P::NBIN < G::NT ? P::NBIN : G::NT), g = P::NBIN < G::NT ? tid / P::NBIN : 0; k < P::NBIN && g < NG2; k += G::NT) {
      // eight loads in flight: each is a round trip to the point of coherence
      float s = 0.0f;
      for (int m = g; m < members; m += 8 * NG2) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = coherent_load(&part[(i64)(m + u * NG2 < members ? m + u * NG2 : m) * P::NBIN + k]);
#pragma unroll
        for (int u = 0; u < 8; ++u) s += m + u * NG2 < members ? q[u] : 0.0f;
      }
      red[g * P::NBIN + k] = s;
    }
    __syncthreads();
    for (int k = tid; k < P::NBIN; k += G::NT) {
      float s = red[k];
      for (int g = 1; g < NG2; ++g) s += red[g * P::NBIN + k];
      P::store_bin(a, row, k, s);
    }
  }
};
