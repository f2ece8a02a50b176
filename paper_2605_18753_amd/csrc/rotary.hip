// Rotary positions of queries and keys, and their inverse for gradients.  C ABI: dash_rotary_turns, dash_rotary_apply.
#include <math.h>

#include "rotary.h"
#include "strided.h"

namespace dash {

struct RotateArgs {
  RotaryArgs r;
  const void* x[2];  void* y[2];         // queries, keys
  const int32_t* pos;
  int64_t pos_b, x_b[2], x_h[2], x_t[2], y_b[2], y_h[2], y_t[2];
  int heads[2], n[2];                    // n: tokens; those of tensor 0 are the last ones
  int tokens, start, inverse;
  uint32_t all;                          // batch * tokens, below 2^31
};

// HBM bounds it where there are many tokens: every byte is read once and written once, 4 x 32 heads of 128 x 8192 tokens in bf16 in 98 us, 5.5 TB/s.  A workgroup has 8 tokens: cosines and sines of
// their pairs are worked out once, into LDS; a thread keeps those of its unit and walks heads.  (The first heads asked for before the cosines, which costs registers
// and so waves: 4 x 32 heads of 128 x 8192 tokens 102 us instead of 97.)
constexpr int kTok = 8;
template <typename T, int D>
__global__ __launch_bounds__(256, 4) void rotary_kernel(RotateArgs a) {
  using U = Unit<T, D>;
  constexpr int SLOTS = 256 / (U::COUNT * kTok);             // heads at a time
  __shared__ float2 cs[kTok][rotary_place(D / 2)];
  const int t = threadIdx.x / U::COUNT % kTok, slot = threadIdx.x / (U::COUNT * kTok) + (int)blockIdx.y * SLOTS, step = SLOTS * (int)gridDim.y;
  const U unit(a.r, threadIdx.x % U::COUNT);
  // a.all tokens of all sequences, one after the other
  for (uint32_t f0 = blockIdx.x * kTok; f0 < a.all; f0 += gridDim.x * kTok) {
    {
      const uint32_t f = min(f0 + (threadIdx.x & (kTok - 1)), a.all - 1), b = f / (uint32_t)a.tokens, j = f - b * a.tokens;
      const int position = (int)((a.pos ? (uint32_t)a.pos[b * a.pos_b + j] : j) + (uint32_t)a.start);
      for (int k = threadIdx.x / kTok; k < a.r.half; k += 256 / kTok) {
        const double2 v = rotary_cos_sin(a.r, a.r.turns[k], position);
        cs[threadIdx.x & (kTok - 1)][rotary_place(k)] = make_float2((float)v.x, (float)(a.inverse ? -v.y : v.y));
      }
    }
    __syncthreads();
    const typename U::Pairs mine = unit.pairs(cs[t]);
    __syncthreads();
    const uint32_t f = f0 + t, b = f / (uint32_t)a.tokens;
    const int j = (int)(f - b * a.tokens);
    if (f >= a.all) break;                                   // the last round: nobody waits any more
    for (int x = 0; x < 2; x++) {
      const int tok = j - (a.tokens - a.n[x]);
      if (!a.x[x] || tok < 0 || (a.x[x] == a.y[x] && !unit.ta && !unit.tb)) continue;
      const T* from = (const T*)a.x[x] + b * a.x_b[x] + tok * a.x_t[x];
      T* to = (T*)a.y[x] + b * a.y_b[x] + tok * a.y_t[x];
      for (int h = slot; h < a.heads[x]; h += step) unit.store(to + h * a.y_h[x], unit.load(from + h * a.x_h[x]), mine, a.r.adjacent);
    }
  }
}

template <typename T, int D> static hipError_t launch_rotary(const RotateArgs& a, hipStream_t st) {
  constexpr int SLOTS = 256 / (Unit<T, D>::COUNT * kTok);
  const int heads = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1];
  const uint32_t groups = (a.all + kTok - 1) / kTok, most = 1u << 20;
  // Few tokens: the heads of a token go to several workgroups, each of which works out the cosines and sines.  (Up to 512 workgroups; without: 1000 tokens of 40
  // heads of 128 8.7 us instead of 7.9; up to 1024: 2 x 20 heads of 64 x 3001 tokens in fp32 12.1 instead of 11.5, by card up to 11.9.)
  const uint32_t split = groups >= 512 ? 1 : (512 + groups - 1) / groups, turns = (uint32_t)(heads + SLOTS - 1) / SLOTS;
  hipLaunchKernelGGL((rotary_kernel<T, D>), dim3(groups < most ? groups : most, split < turns ? split : turns), dim3(256), 0, st, a);
  return hipGetLastError();
}

int rotary_args(const dash_rotary* r, int head_dim, RotaryArgs* out) {
  if (!r || !r->turns || r->reserved != 0 || ((uintptr_t)r->turns & 7) != 0) return DASH_EINVAL;
  if (r->layout != DASH_ROT_HALVES && r->layout != DASH_ROT_ADJACENT) return DASH_EINVAL;
  if (r->rot_dim < 1 || r->rot_dim > head_dim || !((float)r->mscale > 0.f) || !isfinite((float)r->mscale)) return DASH_EINVAL;
  if (r->rot_dim % 16 != 0) return DASH_EUNSUPPORTED;
  *out = {r->turns, r->rot_dim / 2, r->layout == DASH_ROT_ADJACENT, r->mscale};
  return DASH_OK;
}

// The table of turns: 113 bits for a theta, of which the 64 behind the point of theta / (2 pi) count.  (In 64, the power, 2 pi and the division cost up to 0.6 units of
// the last of those for a theta of 1 and 10 for one of 100.)
typedef __float128 Quad;
// 38 digits
static const Quad kTenTo19 = 10000000000000000000ull;
static const Quad kTwoPi = (6283185307179586476ull * kTenTo19 + 9252867665590057684ull) / (kTenTo19 * 1000000000000000000ull);
static const Quad kLnTwo = (6931471805599453094ull * kTenTo19 + 1723212145817656808ull) / (kTenTo19 * kTenTo19);
static Quad quad_exp(Quad x) {                               // the power series of what is left beside a power of two
  const long double k = roundl((long double)(x / kLnTwo));
  const Quad r = x - kLnTwo * k;                             // below 0.35: the 30th term is 2^-153
  Quad sum = 1;
  for (int n = 30; n > 0; n--) sum = 1 + sum * r / n;
  return sum * ldexpl(1.0L, (int)k);
}
static Quad quad_log(double x) {                             // one step of Halley's method: three times the digits
  const Quad y = logl((long double)x), e = quad_exp(y);
  return y + 2 * ((Quad)x - e) / ((Quad)x + e);
}
// x >= 0 without its whole turns, in units of 2^-64, to the nearest
static uint64_t fraction_of(Quad x) {
  int e;
  frexpl((long double)x, &e);
  for (; e >= 0; e--) {
    const Quad bit = ldexpl(1.0L, e);
    if (x >= bit) x -= bit;
  }
  const Quad y = x * 18446744073709551616.0L;
  const uint64_t whole = (uint64_t)y;
  return whole + (y - (Quad)whole >= (Quad)0.5);
}

}  // namespace dash

using namespace dash;

extern "C" {

int dash_rotary_turns(int32_t rot_dim, const double* freq, int32_t scaling, double base, double factor, double original,
                      double low, double high, uint64_t* turns) {
  if (!turns || rot_dim < 16 || rot_dim > 128 || rot_dim % 16 != 0) return DASH_EINVAL;
  const auto positive = [](double x) { return isfinite(x) && x > 0.0; };
  if (!freq) {
    if (scaling < DASH_ROT_PLAIN || scaling > DASH_ROT_PARTS || !positive(base)) return DASH_EINVAL;
    if (scaling != DASH_ROT_PLAIN && !positive(factor)) return DASH_EINVAL;
    if (scaling == DASH_ROT_PARTS && (!positive(original) || !isfinite(low) || !isfinite(high) || !(low < high))) return DASH_EINVAL;
  } else {
    for (int i = 0; i < rot_dim / 2; i++)
      if (!isfinite(freq[i])) return DASH_EINVAL;
  }
  const Quad ln_base = freq ? (Quad)0 : quad_log(base), ln_factor = freq || scaling == DASH_ROT_PLAIN ? (Quad)0 : quad_log(factor);
  uint64_t out[64];
  for (int i = 0; i < rot_dim / 2; i++) {
    Quad theta;
    if (freq) {
      theta = freq[i] < 0 ? -freq[i] : freq[i];
    } else {
      const Quad ln_b = scaling == DASH_ROT_BASE ? ln_base + ln_factor * rot_dim / (rot_dim - 2) : ln_base;
      theta = quad_exp(ln_b * (-2 * i) / rot_dim);
      if (scaling == DASH_ROT_LINEAR) theta /= factor;
      if (scaling == DASH_ROT_PARTS) {
        const Quad c = (theta * original / kTwoPi - low) / ((Quad)high - low), within = c < 0 ? (Quad)0 : c > 1 ? (Quad)1 : c;
        theta *= within + (1 - within) / factor;
      }
    }
    out[i] = fraction_of(theta / kTwoPi);
    if (freq && freq[i] < 0) out[i] = 0 - out[i];
  }
  for (int i = 0; i < rot_dim / 2; i++) turns[i] = out[i];
  return DASH_OK;
}

int dash_rotary_apply(const dash_rotary_params* p, const dash_rotary* r, const int32_t* pos, const void* q, void* q_out,
                      const void* k, void* k_out, void* stream) {
  if (!p || (!q && !k) || !q != !q_out || !k != !k_out) return DASH_EINVAL;
  if (p->batch < 1 || p->head_dim < 1 || (q && (p->h_q < 1 || p->n_q < 1)) || (k && (p->h_kv < 1 || p->n_kv < 1))) return DASH_EINVAL;
  if (p->dtype != DASH_F32 && p->dtype != DASH_BF16) return DASH_EINVAL;
  if ((p->inverse != 0 && p->inverse != 1) || p->reserved != 0 || p->pos_stride < 0 || (q && k && p->n_q > p->n_kv)) return DASH_EINVAL;
  if (p->head_dim != 64 && p->head_dim != 128) return DASH_EUNSUPPORTED;
  RotateArgs a = {};
  if (const int rc = rotary_args(r, p->head_dim, &a.r); rc != DASH_OK) return rc;
  a.x[0] = q; a.x[1] = k; a.y[0] = q_out; a.y[1] = k_out;
  const int64_t* strides[2][2] = {{p->q_stride, p->q_out_stride}, {p->k_stride, p->k_out_stride}};
  const int vec = p->dtype == DASH_BF16 ? 8 : 4;
  for (int x = 0; x < 2; x++) {
    if (!a.x[x]) continue;
    if ((((uintptr_t)a.x[x] | (uintptr_t)a.y[x]) & 15) != 0) return DASH_EINVAL;
    for (int i = 0; i < 3; i++)
      if (strides[x][0][i] < 0 || strides[x][1][i] < 0 || strides[x][0][i] % vec != 0 || strides[x][1][i] % vec != 0 ||
          (a.x[x] == a.y[x] && strides[x][0][i] != strides[x][1][i])) return DASH_EINVAL;
    a.x_b[x] = strides[x][0][0]; a.x_h[x] = strides[x][0][1]; a.x_t[x] = strides[x][0][2];
    a.y_b[x] = strides[x][1][0]; a.y_h[x] = strides[x][1][1]; a.y_t[x] = strides[x][1][2];
    a.heads[x] = x ? p->h_kv : p->h_q;
    a.n[x] = x ? p->n_kv : p->n_q;
  }
  a.tokens = k ? p->n_kv : p->n_q;
  if ((int64_t)p->batch * a.tokens >= (int64_t)1 << 31 || (int64_t)a.heads[0] + a.heads[1] > 1 << 16) return DASH_EUNSUPPORTED;
  // an output has a place for each element, is its input or apart from it, and apart from the other tensor's
  const auto in = [&](int x) { return Strided{a.x[x], 3, {a.x_b[x], a.x_h[x], a.x_t[x]}, {p->batch, a.heads[x], a.n[x]}}; };
  const auto out = [&](int x) { return Strided{a.y[x], 3, {a.y_b[x], a.y_h[x], a.y_t[x]}, {p->batch, a.heads[x], a.n[x]}}; };
  const auto meet = [&](const Strided& x, const Strided& y) { return strided_meet(x, y, p->head_dim, 16 / vec); };
  for (int x = 0; x < 2; x++)
    if (a.x[x] && (strided_repeats(out(x), p->head_dim) || (a.x[x] != a.y[x] && meet(in(x), out(x))))) return DASH_EINVAL;
  if (q && k && (meet(out(0), out(1)) || meet(in(0), out(1)) || meet(out(0), in(1)))) return DASH_EINVAL;
  a.pos = pos; a.pos_b = p->pos_stride; a.start = p->start; a.inverse = p->inverse;
  a.all = (uint32_t)(p->batch * (int64_t)a.tokens);
  const hipStream_t st = (hipStream_t)stream;
  const bool bf = p->dtype == DASH_BF16;
  const hipError_t e = p->head_dim == 128 ? (bf ? launch_rotary<uint16_t, 128>(a, st) : launch_rotary<float, 128>(a, st))
                                          : (bf ? launch_rotary<uint16_t, 64>(a, st) : launch_rotary<float, 64>(a, st));
  return e == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

}  // extern "C"
