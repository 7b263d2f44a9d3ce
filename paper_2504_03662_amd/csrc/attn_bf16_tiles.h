// Tiles of the bf16 attention kernels for one head dimension: their layout in LDS, direct-to-LDS loads and matrix operands.
// Included once per head dimension by the bodies of the kernels, with GX_ATTN_DH defined, inside a namespace of its own.
constexpr int DH = GX_ATTN_DH;         // head dimension of this instantiation (128 or 64)
constexpr int ROWB = DH * 2;           // bytes per tile row
constexpr int CPR = DH / 8;            // 16 B chunks per tile row
static_assert(DH == 128 || DH == 64, "tile swizzles are worked out for these two row lengths");

// 16 B chunk c of tile row r lives at chunk c ^ swz(r), chosen so that both access patterns of a
// tile are free of bank conflicts: ds_read_b128 of 16 consecutive rows at one logical chunk, and
// the transposing read of 4 consecutive rows x 64 B.
//   256 B rows: the low row bits move whole 64 B groups (the 4 rows of a transposing read fall in
//   distinct banks); the next two bits permute inside a group.
//   128 B rows: two rows share a 256 B bank window, so the swizzle depends on r / 2: its low bit
//   flips the 64 B group (rows r and r + 2 of a transposing read), the rest permutes inside it;
//   it is a bijection of (r / 2) % 8 onto the 8 chunks, which keeps 16 consecutive rows distinct.
GX_DEVINL int swz(int r) {
  if (DH == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  const int x = (r >> 1) & 7;
  return ((x & 1) << 2) | (x >> 1);
}

// Direct-to-LDS loads of tiles of ROWS x DH, column blocks of one sample's rows: the buffer ends with the sample's last
// row, so that rows beyond it read as zeros without a comparison, and the column block goes into the instruction's scalar
// offset.  Instruction i of this wave's share of the tile that starts at byte row0_bytes = first row * row bytes.
template <int ROWS, int NW>
struct RowStream {
  static constexpr int RPI = 64 / CPR, PER_WAVE = ROWS / RPI / NW;
  static_assert(PER_WAVE >= 1, "tile too small for the workgroup");
  unsigned voff[PER_WAVE];
  GX_DEVINL void init(int ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < PER_WAVE; i++) {
      const int r = RPI * (wave * PER_WAVE + i) + lane / CPR;
      const int c = (lane % CPR) ^ swz(r);
      voff[i] = (unsigned)(r * ld + c * 8) * 2u;
    }
  }
  GX_DEVINL void issue(__amdgpu_buffer_rsrc_t rsrc, unsigned row0_bytes, int col_bytes, char* dst, int wave, int i) const {
    const unsigned off = voff[i] + row0_bytes;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(dst + (wave * PER_WAVE + i) * 1024), 16, off,
                                             col_bytes, 0, 0);
  }
  GX_DEVINL void load(__amdgpu_buffer_rsrc_t rsrc, unsigned row0_bytes, int col_bytes, char* dst, int wave) const {
#pragma unroll
    for (int i = 0; i < PER_WAVE; i++) issue(rsrc, row0_bytes, col_bytes, dst, wave, i);
  }
};

// MFMA operand whose 32 rows are tile rows r0..r0+31 and whose reduction index is the head
// dimension (step s covers d = 16 s .. 16 s + 15)
GX_DEVINL bf16x8 frag_rows(const char* tile, int r, int s, int g) {
  const int c = (2 * s + g) ^ swz(r);
  return *reinterpret_cast<const bf16x8*>(tile + r * ROWB + (c << 4));
}
// MFMA operands whose 32 rows are head-dim columns 32 dt .. 32 dt + 31 and whose reduction index
// runs over 16 tile rows starting at a multiple of 16, in the slot order of an accumulator column
// (slot (g, e) <-> row 8 (e / 4) + 4 g + e % 4 of the group), come from transposing reads issued
// as untracked asm (see lds_read_tr_issue): the four
// head-dim blocks of the 16 tile rows starting at 16 * GI, from per-lane addresses prepared by
// cols_lane_offsets() plus the tile's LDS address.  The caller waits (lds_wait_le) and pins.
GX_DEVINL void cols_lane_offsets(int lane, unsigned (&off)[2][DH / 32]) {
  const int g = lane >> 5, s = lane & 15, hb = (lane >> 4) & 1;
#pragma unroll
  for (int half = 0; half < 2; half++) {
    const int r = 4 * g + (s >> 2) + 8 * half;       // swz(16 k + r) == swz(r)
#pragma unroll
    for (int dt = 0; dt < DH / 32; dt++) {
      const int d0 = 32 * dt + 16 * hb + 4 * (s & 3);
      off[half][dt] = (unsigned)(r * ROWB + (((d0 >> 3) ^ swz(r)) << 4) + (d0 & 7) * 2);
    }
  }
}
struct ColFrags {
  bf16x4 lo[DH / 32], hi[DH / 32];
};
template <int GI>
GX_DEVINL void cols_issue(unsigned tile, const unsigned (&off)[2][DH / 32], ColFrags& f) {
#pragma unroll
  for (int dt = 0; dt < DH / 32; dt++) {
    f.lo[dt] = lds_read_tr_issue<GI * 16 * ROWB>(tile + off[0][dt]);
    f.hi[dt] = lds_read_tr_issue<GI * 16 * ROWB>(tile + off[1][dt]);
  }
}
GX_DEVINL bf16x8 cols_get(ColFrags& f, int dt) {
  lds_pin(f.lo[dt]);
  lds_pin(f.hi[dt]);
  return __builtin_shufflevector(f.lo[dt], f.hi[dt], 0, 1, 2, 3, 4, 5, 6, 7);
}

// registers v = 8 h .. 8 h + 7 of an accumulator, rounded to bf16, as an MFMA operand
GX_DEVINL bf16x8 pack_half(const f32x16& a, int h) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; e++) o[e] = (bf16)a[8 * h + e];
  return o;
}

GX_DEVINL f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; v++) z[v] = 0.f;
  return z;
}

template <class F, int... I>
GX_DEVINL void unroll_seq(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
// f(0) .. f(N - 1) with the index as a constant
template <int N, class F>
GX_DEVINL void unroll(F&& f) {
  unroll_seq(f, std::make_integer_sequence<int, N>());
}

// N products whose LDS fragments are requested DEPTH products ahead: read(i) returns fragment i, mul(i, f)
// issues product i.  Left to itself the compiler asks for a fragment one product ahead.
template <int N, int DEPTH, class Read, class Mul>
GX_DEVINL void streamed(Read read, Mul mul) {
  bf16x8 f[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH && i < N; i++) f[i] = read(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; i++) {
    mul(i, f[i % DEPTH]);
    __builtin_amdgcn_sched_barrier(0);
    if (i + DEPTH < N) f[i % DEPTH] = read(i + DEPTH);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// this lane's 8 steps of a 32-row operand read straight from global memory (row clamped)
GX_DEVINL void load_row_frags(const bf16* base, int ld, int row, int nrows, int g, bf16x8 (&out)[DH / 16]) {
  const bf16* p = base + (size_t)min(row, nrows - 1) * ld + 8 * g;
#pragma unroll
  for (int s = 0; s < DH / 16; s++) out[s] = *reinterpret_cast<const bf16x8*>(p + 16 * s);
}


// acc[dt] += product of the transposed fragments of a tile of 16 * NG16 rows (groups of 16 rows at LDS address `ct`)
// with xf[group]; rows of the result are head-dim columns.  Groups 0 and 1 must have been issued into cf[0], cf[1] by the
// caller (as early as it likes, to cover LDS latency with its own work); with four groups, groups 2 and 3
// are issued here, so that two groups are always in flight.
template <int NG16>
GX_DEVINL void tr_product(f32x16 (&acc)[DH / 32], unsigned ct, const unsigned (&coff)[2][DH / 32],
                          ColFrags (&cf)[2], const bf16x8 (&xf)[NG16]) {
  static_assert(NG16 == 2 || NG16 == 4, "tiles of 32 or 64 rows");
#define GX_TR_GROUP(U, BUF) \
  _Pragma("unroll") for (int dt = 0; dt < DH / 32; dt++) acc[dt] = MFMA(cols_get(cf[BUF], dt), xf[U], acc[dt])
  lds_wait_le<2 * (DH / 32)>();
  GX_TR_GROUP(0, 0);
  if (NG16 == 4) {
    cols_issue<2>(ct, coff, cf[0]);
    lds_wait_le<2 * (DH / 32)>();
    GX_TR_GROUP(1, 1);
    cols_issue<3>(ct, coff, cf[1]);
    lds_wait_le<2 * (DH / 32)>();
    GX_TR_GROUP(NG16 - 2, 0);
    lds_wait_all();
    GX_TR_GROUP(NG16 - 1, 1);
  } else {
    lds_wait_all();
    GX_TR_GROUP(1, 1);
  }
#undef GX_TR_GROUP
}
