// Entry points of the operators at the end of a training step: the loss of a linear layer over many classes
// (linear_ce.cuh) and the orthogonalised update (ortho.cuh).
#include <math.h>

#include "../../include/lp.h"
#include "gemm_launch.h"
#include "linear_ce.cuh"
#include "ops.h"
#include "ortho.cuh"
#include "ortho_small.cuh"

namespace lp {

// Regions of a scratch buffer, each on a 256-byte boundary.  Without a base it only counts.
struct Carve {
  uint8_t* base;
  size_t off = 0;
  template <typename T>
  T* take(size_t n) {
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += align_up(n * sizeof(T), 256);
    return p;
  }
};
static inline long long row_stride(long long cols) { return (cols + 31) / 32 * 32; }   // whole 32-column groups of the epilogues

// ---------------------------------------------------------------------------------------------
// orthogonalised update
// ---------------------------------------------------------------------------------------------
// Powers of two by which the fp16 planes of X, A and B are larger than the matrices: X's entries are about 1 / sqrt(cols),
// and a low part below 2^-14 would lose bits.  |X| < 16 and |A|, |B| < 63 stay finite.
static const float kScaleX = 4096.f, kScaleA = 1024.f, kScaleB = 1024.f;

struct OrthoScratch {
  int* err;
  float* alpha;
  double* sums;
  __half *x[2], *a, *b;
  int parts;
  long long ld, ld_s;
};
static int ortho_parts(long long elems, int batch) {
  // blocks of at least 4096 elements, about eight an SM over the batch
  const long long want = std::max<long long>(1, 1184 / batch), most = std::max<long long>(1, elems / 4096);
  return (int)std::min<long long>(std::min(want, most), kOrthoMaxParts);
}
static OrthoScratch ortho_carve(Carve& c, int batch, int rows, int cols, bool split) {
  OrthoScratch s;
  const long long small = std::min(rows, cols);
  s.ld = row_stride(cols);
  s.ld_s = row_stride(small);
  s.parts = ortho_parts((long long)rows * cols, batch);
  s.err = c.take<int>(64);
  s.alpha = c.take<float>(batch);
  s.sums = c.take<double>((size_t)batch * s.parts);
  const int planes = split ? 2 : 1;
  for (int i = 0; i < 2; ++i) s.x[i] = c.take<__half>((size_t)2 * batch * rows * s.ld);
  s.a = c.take<__half>((size_t)planes * batch * small * s.ld_s);
  s.b = c.take<__half>((size_t)planes * batch * small * s.ld_s);
  return s;
}
size_t ortho_scratch_bytes(int batch, int rows, int cols, bool split) {
  Carve c{nullptr};
  ortho_carve(c, batch, rows, cols, split);
  return c.off;
}

// One launch for matrices whose X stays in the shared memory of a cluster (ortho_small.cuh): the smaller side is at most 128 and
// the larger fits in 8 slices.  As many CTAs a matrix as keep all clusters resident at once, but slices of 32 columns at least (18
// matrices of 64 x 576: 55 us on clusters of four, 68 on eight, of which 16 fit).
static const size_t kSmallMaxSmem = 224 * 1024;
struct SmallShape { int S, ctas, slice; };
static bool ortho_small_shape(int batch, int rows, int cols, bool split, SmallShape* out) {
  const int s = std::min(rows, cols), l = std::max(rows, cols);
  if (s > 128 || l > (1 << 20)) return false;
  const int S = s <= 16 ? 16 : s <= 32 ? 32 : s <= 64 ? 64 : 128;
  auto slice = [&](int c) { return ((l + c - 1) / c + 15) / 16 * 16; };
  const Device& D = cur_dev();
  int c = 1;
  while (c < 8 && D.small_clusters[2 * c] > 0 &&
         (small_smem(S, slice(c), split) > kSmallMaxSmem || (batch <= D.small_clusters[2 * c] && slice(2 * c) >= 32)))
    c *= 2;
  if (small_smem(S, slice(c), split) > kSmallMaxSmem) return false;
  // (128 rows and more than 64 columns a CTA: 128 x 1152 in fp32 130 us, 122 as products of gemm_tc.cuh; 128 x 512 91 and 112;
  // 40 of 128 x 1152, more than fit at once, 402 and 178; 128 of 64 x 1152, 255 and 216)
  const bool waits = batch > D.small_clusters[c];
  if (S == 128 ? slice(c) > 64 || waits : S == 64 && slice(c) > 288 && waits) return false;
  *out = SmallShape{S, c, slice(c)};
  return true;
}
template <bool kSplit, int S>
static int start_small(const OrthoSmall& p, const SmallShape& sh, int batch, cudaStream_t st) {
  LP_CUDA_OK(launch_pdl_cluster(sh.ctas, ortho_small_kernel<kSplit, S>, dim3((unsigned)(batch * sh.ctas)), dim3(kSmallThreads),
                                small_smem(S, sh.slice, kSplit), st, p));
  return LP_OK;
}
template <int S>
static int small_set_attributes() {
  LP_CUDA_OK(cudaFuncSetAttribute(ortho_small_kernel<true, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallMaxSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(ortho_small_kernel<false, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallMaxSmem));
  return LP_OK;
}
static int ortho_init_dev() {
  int rc = gemm_init_dev();
  if (rc != LP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_devices_mutex);
  Device& D = cur_dev();
  if (D.ortho_attr) return LP_OK;
  if ((rc = small_set_attributes<16>()) != LP_OK || (rc = small_set_attributes<32>()) != LP_OK ||
      (rc = small_set_attributes<64>()) != LP_OK || (rc = small_set_attributes<128>()) != LP_OK)
    return rc;
  for (int c = 1; c <= 8; c *= 2) D.small_clusters[c] = max_clusters(c, ortho_small_kernel<true, 128>, kSmallThreads, kSmallMaxSmem, D.sm_count);
  D.ortho_attr = true;
  return LP_OK;
}
static int ortho_run_small(const OrthoProblem& q, const OrthoSource& src, const SmallShape& sh, int* err, cudaStream_t st) {
  OrthoSmall p;
  memset(&p, 0, sizeof(p));
  p.src = src;
  p.s = std::min(q.rows, q.cols);
  p.l = std::max(q.rows, q.cols);
  p.tall = q.rows > q.cols;
  p.slice = sh.slice; p.ctas = sh.ctas; p.steps = q.steps;
  p.a = q.coeffs[0]; p.b = q.coeffs[1]; p.c = q.coeffs[2]; p.eps = q.eps;
  p.out = q.out; p.out_bf16 = q.out_bf16; p.update = q.update; p.keep = q.keep; p.step = q.step;
  p.err = err;
  switch (sh.S) {
    case 16: return q.split ? start_small<true, 16>(p, sh, q.batch, st) : start_small<false, 16>(p, sh, q.batch, st);
    case 32: return q.split ? start_small<true, 32>(p, sh, q.batch, st) : start_small<false, 32>(p, sh, q.batch, st);
    case 64: return q.split ? start_small<true, 64>(p, sh, q.batch, st) : start_small<false, 64>(p, sh, q.batch, st);
    default: return q.split ? start_small<true, 128>(p, sh, q.batch, st) : start_small<false, 128>(p, sh, q.batch, st);
  }
}

int ortho_run(const OrthoProblem& q, void* scratch, cudaStream_t st, long long* launches) {
  int rc = ortho_init_dev();
  if (rc != LP_OK) return rc;
  const Device& D = cur_dev();
  Carve c{(uint8_t*)scratch};
  OrthoScratch s = ortho_carve(c, q.batch, q.rows, q.cols, q.split);
  int* clear_err = q.err ? nullptr : s.err;
  if (q.err) s.err = q.err;
  if (q.off && q.batch > kOrthoMaxOffsets) return LP_ERR_SIZE;
  const bool tall = q.rows > q.cols;
  const int small = std::min(q.rows, q.cols), B = q.batch;
  const long long x_mat = (long long)q.rows * s.ld, x_plane = B * x_mat, s_mat = (long long)small * s.ld_s, s_plane = B * s_mat;
  const int planes = q.split ? 2 : 1;
  long long n = 0;

  OrthoSource src;
  memset(&src, 0, sizeof(src));
  src.g = q.g; src.g_bf16 = q.g_bf16; src.momentum = q.momentum; src.mu = q.mu; src.nesterov = q.nesterov;
  src.elems = (long long)q.rows * q.cols;
  if (q.off) {
    src.use_off = 1;
    for (int b = 0; b < B; ++b) src.off[b] = q.off[b];
  }
  SmallShape small_shape;
  if (ortho_small_shape(B, q.rows, q.cols, q.split, &small_shape)) {
    if (launches) *launches += 1;
    return ortho_run_small(q, src, small_shape, clear_err, st);
  }
  // (a bf16 gradient is exact in one plane)
  int x_planes = q.split || !q.g_bf16 || q.momentum ? 2 : 1;
  bool flat = B == 1 || src.elems % 8 == 0 || q.off;   // every matrix starts on a group of 8 elements
  for (int b = 0; q.off && b < B; ++b) flat = flat && q.off[b] % 8 == 0;
  const bool vec = flat && q.cols % 8 == 0;
  LP_CUDA_OK(launch_pdl(flat ? ortho_norm_kernel<true> : ortho_norm_kernel<false>, dim3(s.parts, B), dim3(kOrthoThreads), 0, st, src, s.parts,
                        s.sums, clear_err));
  LP_CUDA_OK(launch_pdl(vec ? ortho_pack_kernel<true> : ortho_pack_kernel<false>, dim3(s.parts, B), dim3(kOrthoThreads), 0, st, src, s.parts,
                        (const double*)s.sums, q.eps, q.cols, s.ld, s.x[0], x_mat, x_planes == 2 ? x_plane : 0LL, s.alpha));
  n += 2;

  // tensor maps, once a call: X in both buffers and both orders, A and B with K contiguous (they are symmetric)
  CUtensorMap m_xk[2], m_xm[2], m_a, m_b, m_bh;
  for (int i = 0; i < 2; ++i) {
    const GemmOperand x{s.x[i], q.cols, q.rows, s.ld, x_mat, 2 * B, false};
    if ((rc = encode_gemm_map(&m_xk[i], x, false)) != LP_OK) return rc;
    if ((rc = encode_gemm_map(&m_xm[i], x, true)) != LP_OK) return rc;
  }
  if ((rc = encode_gemm_map(&m_a, GemmOperand{s.a, small, small, s.ld_s, s_mat, planes * B, false}, false)) != LP_OK) return rc;
  if ((rc = encode_gemm_map(&m_b, GemmOperand{s.b, small, small, s.ld_s, s_mat, planes * B, false}, false)) != LP_OK) return rc;
  // (B as the second operand of 256 x 128 tiles)
  const GemmOperand b_half{s.b, small, small, s.ld_s, s_mat, planes * B, false};
  if (tall && q.split && (rc = encode_gemm_map(&m_bh, b_half, false, rows_b(GemmCut{tc::GEMM_HALF, 2}))) != LP_OK) return rc;
  const GemmCut cut_g = gemm_cut(small, small, tall ? q.rows : q.cols, B, true, planes, planes),
                     cut_a = gemm_cut(small, small, small, B, true, planes, planes);

  int cur = 0;
  for (int i = 0; i < q.steps; ++i) {
    const bool first = i == 0, last = i + 1 == q.steps;
    // A = X X^T (X^T X), from the high parts alone unless fp32 results are wanted
    tc::GemmParams p;
    memset(&p, 0, sizeof(p));
    p.M = p.N = small; p.batch = B; p.sym = 1; p.err = s.err;
    p.a_planes = p.b_planes = planes;
    p.f = first ? kScaleA : kScaleA / (kScaleX * kScaleX);
    p.f_dev = s.alpha; p.f_pow = first ? 2 : 0;
    p.h_out = s.a; p.h_ld = s.ld_s; p.h_batch = s_mat; p.h_plane = q.split ? s_plane : 0;
    if (tall) rc = launch_gemm<tc::EPI_H16>(p, q.rows, m_xm[cur], true, m_xm[cur], true, false, cut_g, st);
    else rc = launch_gemm<tc::EPI_H16>(p, q.cols, m_xk[cur], false, m_xk[cur], false, false, cut_g, st);
    if (rc != LP_OK) return rc;
    // B = a I + b A + c A^2
    memset(&p, 0, sizeof(p));
    p.M = p.N = small; p.batch = B; p.sym = 1; p.err = s.err;
    p.a_planes = p.b_planes = planes;
    p.f = q.coeffs[2] * (kScaleB / (kScaleA * kScaleA));
    p.h_out = s.b; p.h_ld = s.ld_s; p.h_batch = s_mat; p.h_plane = q.split ? s_plane : 0;
    p.aux = s.a; p.aux_f = q.coeffs[1] * (kScaleB / kScaleA); p.diag = q.coeffs[0] * kScaleB;
    rc = launch_gemm<tc::EPI_H16>(p, small, m_a, false, m_a, false, false, cut_a, st);
    if (rc != LP_OK) return rc;
    // X <- B X (X B).  An error in X grows by up to a in each later step, so the low part is kept
    // while three or more products follow (relative error, 256 x 2304 of a decaying spectrum: 5.6e-3 without, 1.5e-3 with the
    // low parts of two steps, 1.1e-3 with all; fp16's step in A and B costs 1e-3; a low part costs a product)
    memset(&p, 0, sizeof(p));
    p.M = q.rows; p.N = q.cols; p.batch = B; p.err = s.err;
    p.a_planes = tall ? x_planes : planes;
    p.b_planes = tall ? planes : x_planes;
    p.f = last ? 1.f / (first ? kScaleB : kScaleB * kScaleX) : (first ? kScaleX / kScaleB : 1.f / kScaleB);
    p.f_dev = s.alpha; p.f_pow = first ? 1 : 0;
    const GemmCut cut_x = gemm_cut(q.rows, q.cols, small, B, false, p.a_planes, p.b_planes);
    const CUtensorMap& ma = tall ? m_xk[cur] : m_b;
    const CUtensorMap& mb = !tall ? m_xm[cur] : cut_x.kind == tc::GEMM_HALF ? m_bh : m_b;
    if (last) {
      p.out = q.out; p.out_bf16 = q.out_bf16; p.out_ld = q.cols; p.out_batch = src.elems;
      p.update = q.update; p.keep = q.keep; p.step = q.step;
      if (q.off) {
        p.use_off = 1;
        for (int b = 0; b < B; ++b) p.off[b] = q.off[b];
      }
      rc = launch_gemm<tc::EPI_OUT>(p, small, ma, false, mb, !tall, false, cut_x, st);
    } else {
      x_planes = q.split || i + 3 < q.steps ? 2 : 1;
      cur ^= 1;
      p.h_out = s.x[cur]; p.h_ld = s.ld; p.h_batch = x_mat; p.h_plane = x_planes == 2 ? x_plane : 0;
      rc = launch_gemm<tc::EPI_H16>(p, small, ma, false, mb, !tall, false, cut_x, st);
    }
    if (rc != LP_OK) return rc;
    n += 3;
  }
  if (launches) *launches += n;
  return LP_OK;
}

static_assert(kOrthoMaxOffsets == tc::kGemmMaxOffsets, "one table");
const float kOrthoCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};

// Both parts of everything, for a result in bf16 too where there are few singular values: the roundings of A's and B's diagonals to
// fp16 then move all of them alike, and where the values lie close together the last steps enlarge that up to 20 times (4 and 24 to
// 56 of them: errors of 2.5e-3 to 4e-3 of the norm with bf16's own 1.7e-3; from 64 on 1.8e-3 to 2.8e-3, matrices of equal singular
// values up to 4.3e-3, identities up to 1.02e-2, at 392 rows).  It costs little where latency is what counts (16 x 144 18.0 us and 18.9; 18 x 64 x 576
// would be 39 and 48).
bool ortho_two_parts(int dtype, int rows, int cols) { return dtype == LP_F32 || std::min(rows, cols) < 64; }

static int check_ortho(int dtype, int batch, int rows, int cols, int steps, float eps) {
  if (dtype != LP_F32 && dtype != LP_BF16) return LP_ERR_UNSUPPORTED;
  if (batch < 1 || rows < 1 || cols < 1 || batch > 65535 || steps < 1 || steps > 32) return LP_ERR_SIZE;
  // (sides of 2^24: a product's longest accumulation, 2^18 K blocks, is less than half of what a bounded wait waits)
  if (rows > (1 << 24) || cols > (1 << 24) || std::min(rows, cols) > (1 << 17)) return LP_ERR_SIZE;
  if (!(eps >= 1e-30f) || !(eps <= 1e30f)) return LP_ERR_SIZE;
  return LP_OK;
}

// ---------------------------------------------------------------------------------------------
// loss of a linear layer
// ---------------------------------------------------------------------------------------------
// Exponentials of a piece of rows: 512 MB, or as much as the fp32 sums of dw over several pieces would take, if that makes it
// one piece.
static const size_t kCePieceBytes = (size_t)512 << 20;
static const int kCeAmaxParts = 592;
// K blocks an accumulation (fp32 problems): 24 steps of the tensor core, each of which cuts the sum off by 2^-25 of it on average.  Worst
// gradients of 150 problems, and 1001 x 640 x 20011: one block 4e-7 of the norm and 350 us, two 6e-7 and 327, four 1.5e-6 and 312; plain
// fp32 products 5e-7.
static const int kCeRound = 2;
static const int kCeLongRound = 64;         // and of bf16 logits: each of its 256 steps is cut off, 4096 features 1e-6 of the loss
static const int kCeFewRows = 4;            // the loss alone of so many is one pass over w
static const int kCeFewBlocks = 592;        // four an SM
static const size_t kCeFewSmem = 96 * 1024;

struct CeScratch {
  CeHeader* hdr;
  float *amax, *target, *top, *row_loss, *sums, *acc;
  float2* stats;
  __half *p, *x, *w;
  long long ld_v, ld_d;
  int rows;                        // of a piece
  bool f32, pack_w;
};
static CeScratch ce_carve(Carve& c, int dtype, int T, int D, int V, bool grads) {
  CeScratch s;
  s.f32 = dtype == LP_F32;
  s.pack_w = s.f32 || D % 8;
  const int planes = s.f32 ? 2 : 1;
  s.ld_v = row_stride(V);
  s.ld_d = (D + 7) / 8 * 8;
  // (the loss alone keeps up to 32 bytes for each row and 128 classes)
  const size_t row_bytes = grads ? (size_t)s.ld_v * 2 * planes : (size_t)((V + 127) / 128) * 32;
  const bool whole = grads && !s.f32 && (size_t)T * row_bytes <= (size_t)V * D * 4;
  const long long fit = whole ? T : (long long)(kCePieceBytes / row_bytes) / 256 * 256;
  s.rows = (int)std::min<long long>(T, std::min(std::max(256LL, fit), 1LL << 18));
  s.hdr = c.take<CeHeader>(1);
  s.amax = c.take<float>(2 * kCeAmaxParts);
  s.target = c.take<float>(T);
  s.top = c.take<float>(T);
  s.row_loss = c.take<float>(T);
  // (parts of 32 columns at least; a part a block where a few rows' loss is one pass over w)
  const int tiles32 = 4 * ((V + 127) / 128);
  s.stats = c.take<float2>((size_t)(!grads && T <= kCeFewRows ? std::max(tiles32, kCeFewBlocks) : tiles32) * s.rows);
  const bool pack_x = s.pack_w || grads;
  s.x = pack_x ? c.take<__half>((size_t)planes * T * s.ld_d) : nullptr;
  s.w = s.pack_w ? c.take<__half>((size_t)planes * V * s.ld_d) : nullptr;
  s.p = grads ? c.take<__half>((size_t)planes * s.rows * s.ld_v) : nullptr;
  s.sums = grads ? c.take<float>((size_t)(T / kCeSlab + T / s.rows + 2) * V) : nullptr;
  s.acc = grads && !s.f32 && s.rows < T ? c.take<float>((size_t)V * D) : nullptr;
  return s;
}

// Loss alone of a few rows.
template <typename T, int kRows>
static int start_few(const CeScratch& s, int rows, int D, int V, const T* x, const T* w, const T* bias, const int32_t* labels, int blocks,
                     cudaStream_t st) {
  const size_t smem = (size_t)kRows * D * 4;
  LP_CUDA_OK(launch_pdl(D % VecT<T>::N ? ce_few_kernel<T, kRows, false> : ce_few_kernel<T, kRows, true>, dim3(blocks), dim3(kCeThreads), smem,
                        st, x, w, bias, labels, rows, D, V, s.stats, (long long)s.rows, s.target, s.hdr));
  return LP_OK;
}
template <typename T>
static int ce_few_rows(const CeScratch& s, int rows, int D, int V, const T* x, const T* w, const T* bias, const int32_t* labels, float* row_loss,
                       float* loss, cudaStream_t st) {
  const int blocks = (int)std::min<long long>(std::min(kCeFewBlocks, 4 * cur_dev().sm_count), (V + 31) / 32);
  const int rc = rows == 1 ? start_few<T, 1>(s, rows, D, V, x, w, bias, labels, blocks, st)
                 : rows == 2 ? start_few<T, 2>(s, rows, D, V, x, w, bias, labels, blocks, st)
                             : start_few<T, 4>(s, rows, D, V, x, w, bias, labels, blocks, st);
  if (rc != LP_OK) return rc;
  LP_CUDA_OK(launch_pdl(ce_finish_kernel, dim3(1), dim3(1024), 0, st, (const float2*)s.stats, (long long)s.rows, blocks, rows, V, labels,
                        s.target, s.top, row_loss, loss));
  return LP_OK;
}
template <typename T, int kRows>
static int few_set_attributes() {
  LP_CUDA_OK(cudaFuncSetAttribute(ce_few_kernel<T, kRows, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kCeFewSmem));
  LP_CUDA_OK(cudaFuncSetAttribute(ce_few_kernel<T, kRows, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kCeFewSmem));
  return LP_OK;
}
static int ce_init_dev() {
  int rc = gemm_init_dev();
  if (rc != LP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_devices_mutex);
  Device& D = cur_dev();
  if (D.ce_attr) return LP_OK;
  if ((rc = few_set_attributes<float, 1>()) != LP_OK || (rc = few_set_attributes<float, 2>()) != LP_OK ||
      (rc = few_set_attributes<float, 4>()) != LP_OK || (rc = few_set_attributes<bf16, 1>()) != LP_OK ||
      (rc = few_set_attributes<bf16, 2>()) != LP_OK || (rc = few_set_attributes<bf16, 4>()) != LP_OK)
    return rc;
  D.ce_attr = true;
  return LP_OK;
}

}  // namespace lp

using namespace lp;

extern "C" {

size_t lp_orthogonalize_scratch_bytes(int dtype, int batch, int rows, int cols) {
  if (check_ortho(dtype, batch, rows, cols, 1, 1.f) != LP_OK) return 0;
  return ortho_scratch_bytes(batch, rows, cols, ortho_two_parts(dtype, rows, cols));
}

int lp_orthogonalize(int dtype, int batch, int rows, int cols, const void* g, void* out, int steps, const float* coeffs, float eps,
                     void* scratch, size_t scratch_bytes, void* stream) {
  if (!g || !out || !scratch) return LP_ERR_NULL;
  int rc = check_ortho(dtype, batch, rows, cols, steps, eps);
  if (rc != LP_OK) return rc;
  if (!aligned16(g) || !aligned16(out) || (reinterpret_cast<uintptr_t>(scratch) & 255)) return LP_ERR_ALIGN;
  if (scratch_bytes < lp_orthogonalize_scratch_bytes(dtype, batch, rows, cols)) return LP_ERR_WORKSPACE;
  OrthoProblem q;
  memset(&q, 0, sizeof(q));
  q.batch = batch; q.rows = rows; q.cols = cols;
  q.g_bf16 = q.out_bf16 = dtype == LP_BF16;
  q.split = ortho_two_parts(dtype, rows, cols);
  q.g = g; q.out = out; q.steps = steps; q.eps = eps;
  memcpy(q.coeffs, coeffs ? coeffs : kOrthoCoeffs, sizeof(q.coeffs));
  return ortho_run(q, scratch, (cudaStream_t)stream, nullptr);
}

int lp_muon_update(int dtype, int batch, int rows, int cols, void* w, const void* g, float* momentum_buf, float lr, float momentum,
                   int nesterov, float weight_decay, float scale, int steps, const float* coeffs, float eps, void* scratch,
                   size_t scratch_bytes, void* stream) {
  if (!w || !g || !momentum_buf || !scratch) return LP_ERR_NULL;
  int rc = check_ortho(dtype, batch, rows, cols, steps, eps);
  if (rc != LP_OK) return rc;
  if (!aligned16(w) || !aligned16(g) || !aligned16(momentum_buf) || (reinterpret_cast<uintptr_t>(scratch) & 255)) return LP_ERR_ALIGN;
  if (scratch_bytes < lp_orthogonalize_scratch_bytes(dtype, batch, rows, cols)) return LP_ERR_WORKSPACE;
  OrthoProblem q;
  memset(&q, 0, sizeof(q));
  q.batch = batch; q.rows = rows; q.cols = cols;
  q.g_bf16 = q.out_bf16 = dtype == LP_BF16;
  // (as exact as lp_orthogonalize: rates and weights are the caller's, and beside small or zero weights the step is all there is)
  q.split = ortho_two_parts(dtype, rows, cols);
  q.g = g; q.momentum = momentum_buf; q.mu = momentum; q.nesterov = nesterov != 0;
  q.out = w; q.update = true; q.keep = 1.f - lr * weight_decay; q.step = -lr * scale;
  q.steps = steps; q.eps = eps;
  memcpy(q.coeffs, coeffs ? coeffs : kOrthoCoeffs, sizeof(q.coeffs));
  return ortho_run(q, scratch, (cudaStream_t)stream, nullptr);
}

static bool ce_size_ok(int T, int D, int V) {
  return T >= 1 && D >= 1 && V >= 1 && T <= (1 << 28) && V <= (1 << 24) && D <= (1 << 20);   // (V: see check_ortho)
}

size_t lp_linear_cross_entropy_scratch_bytes(int dtype, int T, int D, int V, int grads) {
  if ((dtype != LP_F32 && dtype != LP_BF16) || !ce_size_ok(T, D, V)) return 0;
  // (what the gradients need is enough for the loss alone: one scratch serves training and evaluation)
  Carve alone{nullptr}, c{nullptr};
  ce_carve(alone, dtype, T, D, V, false);
  if (grads) ce_carve(c, dtype, T, D, V, true);
  return std::max(alone.off, c.off);
}

int lp_linear_cross_entropy(int dtype, int T, int D, int V, const void* x, const void* w, const void* bias, const int32_t* labels,
                            float grad_scale, float* loss_out, float* row_loss, void* dx, void* dw, void* dbias, void* scratch,
                            size_t scratch_bytes, void* stream) {
  if (!x || !w || !labels || !loss_out || !scratch) return LP_ERR_NULL;
  if (dtype != LP_F32 && dtype != LP_BF16) return LP_ERR_UNSUPPORTED;
  if (!ce_size_ok(T, D, V)) return LP_ERR_SIZE;
  const void* ptrs[] = {x, w, bias, labels, loss_out, row_loss, dx, dw, dbias};
  for (const void* p : ptrs)
    if (!aligned16(p)) return LP_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(scratch) & 255) return LP_ERR_ALIGN;
  const bool grads = dx || dw || dbias;
  if (scratch_bytes < lp_linear_cross_entropy_scratch_bytes(dtype, T, D, V, grads)) return LP_ERR_WORKSPACE;
  int rc = ce_init_dev();
  if (rc != LP_OK) return rc;
  const Device& Dv = cur_dev();
  cudaStream_t st = (cudaStream_t)stream;
  Carve c{(uint8_t*)scratch};
  const CeScratch s = ce_carve(c, dtype, T, D, V, grads);
  const int planes = s.f32 ? 2 : 1, is_bf16 = !s.f32;
  const long long x_plane = (long long)T * s.ld_d, w_plane = (long long)V * s.ld_d, p_plane = (long long)s.rows * s.ld_v;
  float* rl = row_loss ? row_loss : s.row_loss;
  if (!grads && T <= kCeFewRows && (size_t)(T == 3 ? 4 : T) * D * 4 <= kCeFewSmem)
    return s.f32 ? ce_few_rows(s, T, D, V, (const float*)x, (const float*)w, (const float*)bias, labels, rl, loss_out, st)
                 : ce_few_rows(s, T, D, V, (const bf16*)x, (const bf16*)w, (const bf16*)bias, labels, rl, loss_out, st);
  if (s.f32)
    LP_CUDA_OK(launch_pdl(ce_prepare_kernel, dim3(1 + 2 * kCeAmaxParts), dim3(kCeThreads), 0, st, labels, T, D, V, (const float*)x, (const float*)w,
                          (const float*)bias, s.amax, kCeAmaxParts, s.hdr));
  if (s.x) {
    const int xb = 1 + grid_for((long long)T * D, kCeThreads * 8, Dv.sm_count, 4);
    const int wb = s.w ? grid_for((long long)V * D, kCeThreads * 8, Dv.sm_count, 8) : 0;
    LP_CUDA_OK(launch_pdl(D % 8 ? ce_pack_kernel<false> : ce_pack_kernel<true>, dim3(xb + wb), dim3(kCeThreads), 0, st, x, w, bias, labels,
                          is_bf16, T, D, V, s.ld_d, s.x, x_plane, s.w, w_plane, xb, (const float*)s.amax, kCeAmaxParts, grad_scale, s.hdr));
  }
  const void* xm = s.x ? (const void*)s.x : x;
  const void* wm = s.w ? (const void*)s.w : w;
  const long long ldx = s.x ? s.ld_d : D, ldw = s.w ? s.ld_d : D;
  CUtensorMap m_wk, m_wm;
  const GemmOperand ow{wm, D, V, ldw, w_plane, planes, !s.f32};
  if ((rc = encode_gemm_map(&m_wm, ow, true)) != LP_OK) return rc;
  int slab0 = 0;
  bool one_slab = false;
  for (int r0 = 0; r0 < T; r0 += s.rows) {
    const int rows = std::min(s.rows, T - r0);
    const GemmOperand ox{(const uint16_t*)xm + (long long)r0 * ldx, D, rows, ldx, x_plane, planes, !s.f32};
    CUtensorMap m_xk, m_xm, m_pk, m_pm;
    if ((rc = encode_gemm_map(&m_xk, ox, false)) != LP_OK) return rc;
    const GemmCut cut = gemm_cut(rows, V, D, 1, false, planes, planes);
    if ((rc = encode_gemm_map(&m_wk, ow, false, rows_b(cut))) != LP_OK) return rc;
    const int part_cols = cut.kind == tc::GEMM_PAIR ? 128 : cut.kind == tc::GEMM_KSPLIT ? 32 : 64;
    const int parts = (V + part_cols - 1) / part_cols;
    tc::GemmParams p;
    memset(&p, 0, sizeof(p));
    p.M = rows; p.N = V; p.batch = 1; p.err = &s.hdr->err;
    p.a_planes = p.b_planes = planes;
    p.f = 1.f; p.f_dev = &s.hdr->logit_f; p.f_pow = s.f32 ? 1 : 0;
    p.bias = bias; p.bias_bf16 = is_bf16; p.labels = labels + r0;
    p.stats = s.stats; p.stats_ld = s.rows; p.target = s.target + r0;
    p.h_out = s.p; p.h_ld = s.ld_v; p.h_plane = s.f32 ? p_plane : 0;
    p.round_len = s.f32 ? kCeRound : kCeLongRound;
    if (!s.x && r0 == 0) p.clear = &s.hdr->err;   // (no kernel before that could have)
    if ((rc = launch_gemm<tc::EPI_CE>(p, D, m_xk, false, m_wk, false, !s.f32, cut, st)) != LP_OK) return rc;
    // few rows and parts: one block does the rest of the loss (us with it and without: 16 x 512 x 4000 in fp32, the loss alone, 23.0 and
    // 24.1; 64 x 512 x 1000 with gradients 39.4 and 38.9; in bf16 the loss alone of 256 rows or of 500 parts 22 or 18 and 15)
    const bool finished = rows == T && rows <= 64 && parts <= 128;
    if (finished)
      LP_CUDA_OK(launch_pdl(ce_finish_kernel, dim3(1), dim3(1024), 0, st, (const float2*)s.stats, (long long)s.rows, parts, rows, V, labels,
                            s.target, s.top, rl, loss_out));
    else
      LP_CUDA_OK(launch_pdl(ce_rows_kernel, dim3((rows + 7) / 8), dim3(kCeThreads), 0, st, (const float2*)s.stats, (long long)s.rows, parts,
                            r0, rows, T, V, labels, s.target, s.top, rl, s.hdr, r0 + rows == T ? loss_out : nullptr));
    if (!grads) continue;
    const int slabs = (rows + kCeSlab - 1) / kCeSlab;
    one_slab = slabs == 1 && rows == T;
    float* sums = dbias && !one_slab ? s.sums + (long long)slab0 * V : nullptr;
    LP_CUDA_OK(launch_pdl(s.f32 ? ce_dl_kernel<true> : ce_dl_kernel<false>, dim3((V + 255) / 256, slabs), dim3(kCeThreads), 0, st, s.p, s.ld_v,
                          p_plane, rows, V, (const float2*)s.stats, (long long)s.rows, part_cols, (const float*)(s.top + r0),
                          (const float*)(s.target + r0), (const float*)(rl + r0), labels + r0, sums, one_slab ? dbias : nullptr, (const CeHeader*)s.hdr));
    slab0 += slabs;
    bool dx_idle = false;
    const GemmOperand op{s.p, V, rows, s.ld_v, p_plane, planes, !s.f32};
    if (dx) {
      if ((rc = encode_gemm_map(&m_pk, op, false)) != LP_OK) return rc;
      memset(&p, 0, sizeof(p));
      p.M = rows; p.N = D; p.batch = 1; p.err = &s.hdr->err;
      p.a_planes = p.b_planes = planes;
      p.f = 1.f; p.f_dev = &s.hdr->dx_f; p.f_pow = 1;
      p.out = (uint8_t*)dx + (size_t)r0 * D * esize(dtype); p.out_bf16 = is_bf16; p.out_ld = D;
      p.labels = labels + r0; p.classes = V;   // (0 * inf of w must not reach a row that does not count)
      const GemmCut kd = gemm_cut(rows, D, V, 1, false, planes, planes);
      p.round_len = s.f32 ? kCeRound : 0;
      p.publish = &s.hdr->dl_seen; p.turn = r0 / s.rows + 1;
      if ((rc = launch_gemm<tc::EPI_OUT>(p, V, m_pk, false, m_wm, true, !s.f32, kd, st)) != LP_OK) return rc;
      dx_idle = p.total_tiles * kd.ctas < Dv.sm_count;
    }
    if (dw) {
      if ((rc = encode_gemm_map(&m_pm, op, true)) != LP_OK) return rc;
      if ((rc = encode_gemm_map(&m_xm, ox, true)) != LP_OK) return rc;
      memset(&p, 0, sizeof(p));
      p.M = V; p.N = D; p.batch = 1; p.err = &s.hdr->err;
      p.a_planes = p.b_planes = planes;
      p.f = 1.f; p.f_dev = &s.hdr->dw_f; p.f_pow = 1;
      p.out = dw; p.out_bf16 = is_bf16; p.out_ld = D;
      // (beside dx's product where that leaves SMs idle: 64 rows x 512 x 1000 28.5 us and 30.5 one after the other, fp32 39.5 and 45;
      // where it has all of them the two share L2 badly, 4096 x 2048 x 32000 1.32 ms and 1.31)
      p.wait_late = dx_idle ? &s.hdr->dl_seen : nullptr; p.turn = r0 / s.rows + 1;
      if (s.rows < T) {
        p.acc = s.f32 ? (float*)dw : s.acc;
        p.acc_first = r0 == 0;
        p.acc_last = r0 + rows == T;
      }
      const GemmCut kd = gemm_cut(V, D, rows, 1, false, planes, planes);
      p.round_len = s.f32 ? kCeRound : 0;
      if ((rc = launch_gemm<tc::EPI_OUT>(p, rows, m_pm, true, m_xm, true, !s.f32, kd, st)) != LP_OK) return rc;
    }
  }
  if (dbias && !one_slab)
    LP_CUDA_OK(launch_pdl(ce_dbias_kernel, dim3((V + kCeThreads - 1) / kCeThreads), dim3(kCeThreads), 0, st, (const float*)s.sums, slab0, V,
                          (const CeHeader*)s.hdr, dbias, is_bf16));
  return LP_OK;
}

int lp_scratch_status(const void* scratch, void* stream) {
  if (!scratch) return LP_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(scratch) & 255) return LP_ERR_ALIGN;
  LP_CUDA_OK(cudaStreamSynchronize((cudaStream_t)stream));
  int e = 0;
  LP_CUDA_OK(cudaMemcpy(&e, scratch, sizeof(e), cudaMemcpyDeviceToHost));
  return e ? LP_ERR_DEVICE_TIMEOUT : LP_OK;
}

}  // extern "C"
