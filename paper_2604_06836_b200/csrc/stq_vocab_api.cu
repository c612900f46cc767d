// C-ABI host layer of the vocabulary cross entropy: argument checks, workspace, launches.
#include "stq_checks.h"
#include "stq_q8.h"
#include "stq_q8_tma.h"
#include "stq_vocab.h"

using namespace stq;

namespace {

constexpr uint32_t kTokensAtOnce = 32768;       // of a loss, at most (tokens do not depend on one another), and
constexpr size_t kPartBytes = 256u << 20;       // of its parts: together they bound its workspace
constexpr size_t kPieceBytes = 512u << 20;      // of gradients of logits that exist at a time

size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// Places in the workspace, one after the other; the first pass only adds up.
struct Arena {
  uint8_t* base = nullptr;
  size_t at = 0;
  template <class T>
  T* take(size_t count) {
    T* p = base ? reinterpret_cast<T*>(base + at) : nullptr;
    at += up(count * sizeof(T), 256);
    return p;
  }
};

// Rows of x that the products can read: those of tokens that count, aligned, or x as it is.
struct Rows {
  bool gather, pitch_w;
  uint16_t *x, *w;
  size_t ldx, ldw;
  uint32_t *count, *token;
  int32_t* row;
  float* scale;

  Rows(const VocabArgs& a, const void* x_, size_t ldx_, bool backward) {
    // For a loss of up to one tile of tokens there is nothing to gain from leaving some out.  (For dw there is: what a token
    // without a loss holds may be NaN, and its product with 0 too.)
    gather = backward || a.t > 256 || !rows_aligned(x_, a.t > 1 ? ldx_ * 2 : 0);
    pitch_w = !rows_aligned(a.w, a.v > 1 ? a.ldw * 2 : 0);
    ldx = up(a.d, 8);
    ldw = up(a.d, 8);
  }
  void place(Arena& m, const VocabArgs& a, uint32_t most) {
    x = gather ? m.take<uint16_t>(most * ldx) : nullptr;
    count = gather ? m.take<uint32_t>(1) : nullptr;
    token = gather ? m.take<uint32_t>(most) : nullptr;
    row = gather ? m.take<int32_t>(a.t) : nullptr;
    scale = gather ? m.take<float>(1) : nullptr;
    w = pitch_w ? m.take<uint16_t>((size_t)a.v * ldw) : nullptr;
  }
};

uint32_t most_rows(uint32_t t) { return t <= 128 ? 128 : (uint32_t)up(t, 256); }

// Sets a.r (and the aligned copy of w) up on the stream.
// (dloss: for the gradients)
cudaError_t prepare_rows(VocabArgs& a, Rows& r, const void* x, size_t ldx, const float* dloss, bool with_w, cudaStream_t s, int* launches) {
  const uint32_t most = most_rows(a.t);
  a.r = {x, a.t > 1 ? ldx : up(a.d, 8), a.t, most, nullptr, nullptr, nullptr, nullptr};
  if (r.gather) {
    const GatherArgs g = {x, ldx, a.t, a.d, most, a.target, a.ignore, r.x, r.ldx, r.count, r.token, r.row, dloss,
                          dloss ? r.scale : nullptr, false};
    const cudaError_t e = launch_vocab_gather(g, s);
    if (e != cudaSuccess) return e;
    a.r = {r.x, r.ldx, most, most, r.count, r.token, r.row, r.scale};
    ++*launches;
  }
  if (r.pitch_w && with_w) {
    const cudaError_t e = launch_pitch(a.w, a.ldw, a.v, a.d, r.w, r.ldw, s);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  if (r.pitch_w) {
    a.w = r.w;
    a.ldw = r.ldw;
  } else if (a.v == 1) {
    a.ldw = up(a.d, 8);
  }
  return cudaSuccess;
}

// Entries of the vocabulary to a piece (the last piece has what is left): as many tiles as fit, or somewhat fewer where the tiles of the
// products then fill their last round better, by half a percent at least: each piece is another beginning and end of dx too, which the
// cost leaves out (8192 x 768 x 50257, fp32 dw: five pieces 3068 us, six, that cost 0.2 % less by the sums below, 3109).
uint32_t piece_of(const VocabArgs& a, VocabDw g, int planes, bool dw, int sms) {
  const uint32_t tiles = (uint32_t)(up(a.v, 256) / 256);
  const size_t fit = kPieceBytes / ((size_t)g.r.most * 2 * planes) / 256;
  if (fit >= tiles) return a.v;
  const uint32_t widest = fit < 1 ? 1 : (uint32_t)fit;
  auto cost = [&](uint32_t cols) {
    double c, extra = 60000.0;      // (of a piece: launches, beginnings and ends)
    vocab_shape(a.t, cols, a.d, planes, sms, &c);
    g.cols = cols;
    return c + extra + (dw ? vocab_dw_cost(g, sms) : 0.0);
  };
  uint32_t best = widest;
  double least = 1e300;
  for (uint32_t w = widest; w > widest - widest / 3 && w > 0; --w) {
    const uint32_t last = a.v - (tiles - 1) / w * w * 256;
    const double c = ((tiles - 1) / w) * cost(w * 256) + cost(last);
    if (c < 0.995 * least) { least = c; best = w; }
  }
  return best * 256;
}

int check(const stq_handle* h, const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias, const int64_t* target, uint64_t t,
          uint32_t v, uint32_t d) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_size(t, d));
  STQ_TRY(check_size(t, v));
  if (t > STQ_VOCAB_MAX_TOKENS || d > STQ_VOCAB_MAX_WIDTH) return STQ_E_TOO_LARGE;
  if (t == 0) return STQ_OK;
  STQ_TRY(check_mat(x, ldx, d, 2));
  STQ_TRY(check_mat(w, ldw, d, 2));
  if (!target) return STQ_E_NULL;
  return aligned(target, 8) && aligned(bias, 4) ? STQ_OK : STQ_E_ALIGN;
}

}  // namespace

extern "C" {

int stq_vocab_loss(stq_handle* h, const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias, const int64_t* target,
                   int64_t ignore_index, uint64_t t, uint32_t v, uint32_t d, float* loss, float* lse, void* stream) {
  STQ_TRY(check(h, x, ldx, w, ldw, bias, target, t, v, d));
  if (t == 0) return STQ_OK;
  if (!loss || !lse) return STQ_E_NULL;
  if (!aligned(loss, 4) || !aligned(lse, 4)) return STQ_E_ALIGN;
  const Span out[] = {{loss, t * 4}, {lse, t * 4}};
  const Span in[] = {mat(x, ldx, t, d, 2), mat(w, ldw, v, d, 2), {bias, v * 4ull}, {target, t * 8}};
  if (clash(out, in)) return STQ_E_ALIAS;
  STQ_CUDA(h, cudaSetDevice(h->device));
  cudaStream_t s = static_cast<cudaStream_t>(stream);

  VocabArgs a = {};
  a.w = w; a.ldw = ldw; a.bias = bias;
  a.v = v; a.d = d;
  a.ignore = ignore_index;
  a.device = h->device;
  // (the blocks of tokens share one workspace, laid out for the largest; tiles of so many entries are 128 wide at least)
  const size_t fit = kPartBytes / (8 * vocab_parts_of_tile(d) * (up(v, 128) / 128)) / 256 * 256;
  const uint32_t at_once = fit < 256 ? 256 : fit < kTokensAtOnce ? (uint32_t)fit : kTokensAtOnce;
  a.t = (uint32_t)(t < at_once ? t : at_once);
  a.target = target;
  Rows r(a, x, ldx, false);
  const uint32_t most = most_rows(a.t);
  const VocabShape shape = vocab_shape(a.t, v, d, 0, h->sm_count);
  const uint32_t parts = vocab_parts(a, shape, most, h->sm_count);
  Arena m;
  float2* part = nullptr;
  float* chosen = nullptr;
  for (int pass = 0; pass < 2; ++pass) {
    m.at = 0;
    r.place(m, a, most);
    part = m.take<float2>((size_t)parts * most);
    chosen = m.take<float>(most);
    if (pass == 0) STQ_TRY(workspace(h, m.at, s, &m.base));
  }
  for (uint64_t t0 = 0; t0 < t; t0 += at_once) {
    VocabArgs b = a;
    b.t = (uint32_t)(t - t0 < at_once ? t - t0 : at_once);
    b.target = target + t0;
    const uint16_t* xb = static_cast<const uint16_t*>(x) + t0 * ldx;
    int launches = 2;
    STQ_CUDA(h, prepare_rows(b, r, xb, ldx, nullptr, t0 == 0, s, &launches));
    STQ_CUDA(h, launch_vocab_parts(b, shape, most, part, chosen, h->sm_count, h->d_err, s));
    STQ_CUDA(h, launch_vocab_finish(b, part, parts, chosen, loss + t0, lse + t0, h->sm_count, s));
    h->launches += launches;
  }
  return STQ_OK;
}

int stq_vocab_loss_backward(stq_handle* h, const float* dloss, const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias,
                            const int64_t* target, int64_t ignore_index, const float* lse, uint64_t t, uint32_t v, uint32_t d, void* dx,
                            uint64_t lddx, void* dw, uint64_t lddw, int dw_dtype, float* dbias, void* stream) {
  STQ_TRY(check(h, x, ldx, w, ldw, bias, target, t, v, d));
  STQ_TRY(check_dtype(dw_dtype));
  const size_t e = elem(dw_dtype);
  if (dw) STQ_TRY(check_mat(dw, lddw, d, e));
  if (!aligned(dbias, 4)) return STQ_E_ALIGN;
  STQ_CUDA(h, cudaSetDevice(h->device));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) {
    if (dw) STQ_TRY(zero(h, dw, lddw, v, d, e, s));
    if (dbias) STQ_TRY(zero(h, dbias, v, 1, v, 4, s));
    return STQ_OK;
  }
  if (dx) STQ_TRY(check_mat(dx, lddx, d, 2));
  if (!dloss || !lse) return STQ_E_NULL;
  if (!aligned(dloss, 4) || !aligned(lse, 4)) return STQ_E_ALIGN;
  const Span out[] = {mat(dx, lddx, t, d, 2), mat(dw, lddw, v, d, e), {dbias, v * 4ull}};
  const Span in[] = {mat(x, ldx, t, d, 2), mat(w, ldw, v, d, 2), {bias, v * 4ull}, {target, t * 8}, {dloss, t * 4}, {lse, t * 4}};
  if (clash(out, in)) return STQ_E_ALIAS;
  if (!dx && !dw && !dbias) return STQ_OK;

  VocabArgs a = {};
  a.w = w; a.ldw = ldw; a.bias = bias;
  a.v = v; a.d = d;
  a.t = (uint32_t)t;
  a.target = target;
  a.ignore = ignore_index;
  a.device = h->device;
  Rows r(a, x, ldx, true);
  const uint32_t most = most_rows(a.t);
  const int planes = dw && dw_dtype == STQ_GRAD_F32 ? 3 : 1;
  VocabDw gw = {};
  gw.dw = dw;
  gw.d = d;
  gw.lddw = lddw;
  gw.f32 = dw_dtype == STQ_GRAD_F32;
  gw.device = h->device;
  gw.r.most = most;
  const uint32_t cols = piece_of(a, gw, planes, dw != nullptr, h->sm_count);
  VocabGradOut o = {nullptr, (uint32_t)(up(cols, 64) / 64), planes, nullptr, 0, lse, dloss};
  gw.panels = o.panels;
  gw.cols = cols;
  // sums for dbias: of the whole vocabulary, if that is not too much, and joined once; else piece by piece
  const size_t db_rows = most / 32;
  const bool db_once = db_rows * up(v, 64) * 4 <= kPieceBytes / 8;
  o.ldb = db_once ? up(v, 64) : up(cols, 64);
  VocabDx gx = {};
  gx.panels = o.panels;
  gx.d = d; gx.first = cols;
  gx.ldd = up(d, 32);
  gx.device = h->device;
  size_t plane = 0, segments = 0;
  vocab_dx_space(most, d, gx.ldd, h->sm_count, &plane, &segments);
  // (a last piece may share its tiles in another way than the others)
  const uint32_t last = (uint32_t)(v - (v - 1) / cols * cols);
  size_t partial = dw ? vocab_dw_partial(gw, h->sm_count) : 0;
  if (dw && last != cols) {
    VocabDw l = gw;
    l.cols = last;
    const size_t p = vocab_dw_partial(l, h->sm_count);
    if (p > partial) partial = p;
  }
  Arena m;
  float *part = nullptr, *db_part = nullptr;
  for (int pass = 0; pass < 2; ++pass) {
    m.at = 0;
    r.place(m, a, most);
    o.p = m.take<uint16_t>((size_t)most * planes * o.panels * 64);
    db_part = dbias ? m.take<float>(db_rows * o.ldb) : nullptr;
    part = partial ? m.take<float>(partial) : nullptr;
    gx.plane = dx ? m.take<float>(plane) : nullptr;
    gx.segments = dx ? m.take<float>(segments) : nullptr;
    if (pass == 0) STQ_TRY(workspace(h, m.at, s, &m.base));
  }
  int launches = 0;
  STQ_CUDA(h, prepare_rows(a, r, x, ldx, dloss, true, s, &launches));
  gw.r = gx.r = a.r;
  gw.p = gx.p = o.p;
  gx.ldw = a.ldw;
  for (uint32_t v0 = 0; v0 < v; v0 += cols) {
    const uint32_t n = v - v0 < cols ? v - v0 : cols;
    o.dbias = db_part && db_once ? db_part + v0 : db_part;
    STQ_CUDA(h, launch_vocab_dlogits(a, vocab_shape(a.t, n, d, planes, h->sm_count), v0, v0 + n, o, h->sm_count, h->d_err, s));
    ++launches;
    if (dbias && !db_once) {
      STQ_CUDA(h, launch_vocab_dbias({db_part, o.ldb, n, dbias + v0}, a.r, s));
      ++launches;
    }
    if (dw) {
      gw.cols = n;
      gw.dw = static_cast<uint8_t*>(dw) + (size_t)v0 * lddw * e;
      STQ_CUDA(h, launch_vocab_dw(gw, part, h->sm_count, h->d_err, s));
      ++launches;
    }
    if (dx) {
      gx.cols = n;
      gx.begin = v0 == 0;
      gx.beside = dw != nullptr;
      gx.w = static_cast<const uint16_t*>(a.w) + (size_t)v0 * a.ldw;
      STQ_CUDA(h, launch_vocab_dx(gx, h->sm_count, h->d_err, s));
      ++launches;
    }
    if (dw) STQ_CUDA(h, launch_vocab_dw_join(gw, part, h->sm_count, s, &launches));
  }
  const VocabDbias db = {db_part, o.ldb, v, dbias};
  const bool join_db = dbias && db_once;
  if (dx) STQ_CUDA(h, launch_vocab_dx_finish(gx, a.t, dx, lddx, join_db ? &db : nullptr, h->sm_count, s));
  else if (join_db) STQ_CUDA(h, launch_vocab_dbias(db, a.r, s));
  if (dx || join_db) ++launches;
  h->launches += launches;
  return STQ_OK;
}

}  // extern "C"
