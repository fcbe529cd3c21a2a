// Log-probabilities of given tokens with entropy and the most likely alternatives, and their gradient with respect to the logits.
//
// With mx the row's largest logit, e_v = exp((z_v - mx)/T), S = sum e and E = sum e (mx - z)/T:
//   ln p_v = (z_v - mx)/T - ln S,   entropy = ln S + E / S,
//   dz_v = (1/T) [ sum over tokens of v of g - p_v (G + gH (ln p_v + entropy)) ],   G = sum of the row's g.
#include <math.h>

#include "device_math.h"
#include "otv_host.h"

namespace otv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNan = __builtin_nanf("");

struct LogprobArgs {
  ot_logprob_in in;
  ot_logprob_out out;
};

__device__ inline float logit(const void* row, int dtype, int64_t v) {
  return dtype == OT_BF16 ? bf16_to_f32(static_cast<const uint16_t*>(row)[v]) : static_cast<const float*>(row)[v];
}
__device__ inline const void* row_of(const ot_logprob_in& in, int64_t row) {
  return static_cast<const char*>(in.logits) + row * in.ld * (in.dtype == OT_BF16 ? 2 : 4);
}
// Temperature of a row, of which log2(e) / T is finite; by a whole wavefront.
__device__ inline float row_temperature(const ot_logprob_in& in, int row, int lane) {
  if (!in.temperature) return 1.f;
  const float T = in.temperature[in.row_off ? find_sequence(in.row_off, in.B, row, 0, lane) : row];
  return T > 0.f ? fmaxf(T, 0x1p-126f) : 1.f;
}
__device__ inline bool any_given(const ot_logprob_in& in, int64_t row) {
  for (int i = 0; i < in.n_tok; ++i)
    if (in.tokens[row * in.n_tok + i] != -1) return true;
  return false;
}

// Order of alternatives as one number: by descending logit (-0 and 0 alike), of equal ones the lowest id first; 0 is none.
__device__ inline unsigned long long order_key(float z, int v) {
  const uint32_t u = __float_as_uint(z + 0.f), up = u & 0x80000000u ? ~u : u | 0x80000000u;
  return z > -INFINITY ? (unsigned long long)up << 32 | (0xFFFFFFFFu - (uint32_t)v) : 0ull;
}
__device__ inline unsigned long long wave_max(unsigned long long k) {
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned long long other = __shfl_xor(k, o);
    k = other > k ? other : k;
  }
  return k;
}

// One workgroup per row.
__global__ __launch_bounds__(256) void logprob_kernel(LogprobArgs a) {
  const ot_logprob_in& in = a.in;
  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ float s_f[4];
  __shared__ double s_d[2][4];
  __shared__ unsigned long long s_k[4];
  const void* z = row_of(in, row);
  const float T = row_temperature(in, row, lane);
  const float scale = kLog2e / T;
  const bool skip = in.given_rows_only && !any_given(in, row);
  const int V = skip ? 0 : in.V;
  float mx = -INFINITY;
  for (int v = tid; v < V; v += 256) mx = fmaxf(mx, logit(z, in.dtype, v));
  mx = otv::wave_max(mx);
  if (lane == 0) s_f[wave] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(s_f[0], s_f[1]), fmaxf(s_f[2], s_f[3]));
  const float top = mx == -INFINITY ? 0.f : mx;
  double S = 0.0, E = 0.0;
  for (int v = tid; v < V; v += 256) {
    const float t = (logit(z, in.dtype, v) - top) * scale, e = __builtin_amdgcn_exp2f(t);
    S += e;
    E -= e * fmaxf(t, -200.f);
  }
  S = wave_sum(S); E = wave_sum(E);
  if (lane == 0) { s_d[0][wave] = S; s_d[1][wave] = E; }
  __syncthreads();
  S = s_d[0][0] + s_d[0][1] + s_d[0][2] + s_d[0][3];
  E = s_d[1][0] + s_d[1][1] + s_d[1][2] + s_d[1][3];
  const double lnS = log(S);
  const float invalid = S == 0.0 ? -INFINITY : kNan;      // of a row without a distribution
  const bool valid = S > 0.0 && S < 1e300;
  if (tid == 0) {
    if (a.out.entropy) a.out.entropy[row] = valid ? (float)(lnS + E / S * 0.6931471805599453) : S == 0.0 ? 0.f : kNan;
    if (a.out.row_max) { a.out.row_max[row] = mx; a.out.row_sumexp[row] = valid || S == 0.0 ? (float)S : kNan; }
  }
  for (int i = tid; i < in.n_tok; i += 256) {
    const int t = in.tokens[(int64_t)row * in.n_tok + i];
    float lp = 0.f;
    if (t < -1 || t >= in.V) lp = kNan;
    else if (t >= 0) lp = valid ? (float)(((double)logit(z, in.dtype, t) - (double)mx) / (double)T - lnS) : invalid;
    a.out.logprob[(int64_t)row * in.n_tok + i] = lp;
  }
  unsigned long long below = ~0ull;
  for (int n = 0; n < in.n_top; ++n) {
    unsigned long long best = 0;
    if (valid)
      for (int v = tid; v < V; v += 256) {
        const unsigned long long k = order_key(logit(z, in.dtype, v), v);
        if (k < below && k > best) best = k;
      }
    best = wave_max(best);
    __syncthreads();
    if (lane == 0) s_k[wave] = best;
    __syncthreads();
    for (int w = 0; w < 4; ++w) best = s_k[w] > best ? s_k[w] : best;
    if (tid == 0) {
      const int id = best ? (int)(0xFFFFFFFFu - (uint32_t)best) : -1;
      a.out.top_ids[(int64_t)row * in.n_top + n] = id;
      a.out.top_logprobs[(int64_t)row * in.n_top + n] =
          best ? (float)(((double)logit(z, in.dtype, id) - (double)mx) / (double)T - lnS) : -INFINITY;
    }
    below = best ? best : 0;
  }
}

struct LogprobGradArgs {
  ot_logprob_in in;
  const float *row_max, *row_sumexp, *entropy, *grad_logprob, *grad_entropy;
  void* grad;
  int64_t ld_grad;
};

__device__ inline uint16_t f32_to_bf16(float x) {         // to nearest, ties to even; NaN stays one
  const uint32_t u = __float_as_uint(x);
  return x != x ? 0x7FC0 : (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}

// Grid = chunks x rows.
constexpr int kGradChunk = 2048;
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobGradArgs a, int chunks) {
  const ot_logprob_in& in = a.in;
  const int row = blockIdx.x / chunks, v0 = (int)(blockIdx.x % chunks) * kGradChunk, tid = threadIdx.x, lane = tid & 63;
  const void* z = row_of(in, row);
  const float T = row_temperature(in, row, lane), scale = kLog2e / T, invT = 1.f / T;
  const float mx = a.row_max[row], S = a.row_sumexp[row];
  const float lnS = logf(S), invS = 1.f / S, gH = a.grad_entropy ? a.grad_entropy[row] : 0.f, H = a.grad_entropy ? a.entropy[row] : 0.f;
  float G = 0.f;
  for (int i = 0; a.grad_logprob && i < in.n_tok; ++i) {
    const int t = in.tokens[(int64_t)row * in.n_tok + i];
    if (t >= 0 && t < in.V) G += a.grad_logprob[(int64_t)row * in.n_tok + i];
  }
  for (int v = v0 + tid; v < min(v0 + kGradChunk, in.V); v += 256) {
    float out = 0.f;
    if (S != 0.f) {
      const float x = logit(z, in.dtype, v), t = (x - mx) * scale, p = __builtin_amdgcn_exp2f(t) * invS;
      const float lp = fmaxf(t, -200.f) * 0.69314718f - lnS;
      out = -p * (G + gH * (lp + H));
      for (int i = 0; a.grad_logprob && i < in.n_tok; ++i)
        if (in.tokens[(int64_t)row * in.n_tok + i] == v && x > -INFINITY) out += a.grad_logprob[(int64_t)row * in.n_tok + i];
      out *= invT;
    }
    const int64_t at = (int64_t)row * a.ld_grad + v;
    if (in.dtype == OT_BF16) static_cast<uint16_t*>(a.grad)[at] = f32_to_bf16(out);
    else static_cast<float*>(a.grad)[at] = out;
  }
}

int check_in(const ot_ctx* ctx, const ot_logprob_in* in, const char* who) {
  if (in->dtype != OT_BF16 && in->dtype != OT_F32) return ot_fail(OT_ERR_DTYPE, "%s: logits are OT_BF16 or OT_F32 (%d)", who, in->dtype);
  if (in->M < 0 || in->V < 1 || in->n_tok < 0 || in->ld < in->V)
    return ot_fail(OT_ERR_SHAPE, "%s: need M >= 0, V >= 1, n_tok >= 0 and ld >= V (M = %d, V = %d, n_tok = %d, ld = %lld)", who, in->M, in->V, in->n_tok, (long long)in->ld);
  if (in->n_top < 0 || in->n_top > OT_MAX_TOP) return ot_fail(OT_ERR_SHAPE, "%s: n_top must be in 0..%d (%d)", who, OT_MAX_TOP, in->n_top);
  if (in->reserved != 0) return ot_fail(OT_ERR_SHAPE, "%s: reserved must be 0", who);
  if (in->given_rows_only && in->n_tok == 0) return ot_fail(OT_ERR_SHAPE, "%s: given_rows_only needs tokens", who);
  if (in->row_off && (in->B < 1 || !in->temperature)) return ot_fail(OT_ERR_SHAPE, "%s: row_off needs B >= 1 sequences and their temperatures", who);
  if (in->M > 0 && (!in->logits || (in->n_tok > 0 && !in->tokens))) return ot_fail(OT_ERR_NULL, "%s: logits and tokens must not be NULL", who);
  if (reinterpret_cast<uintptr_t>(in->logits) % (in->dtype == OT_BF16 ? 2 : 4)) return ot_fail(OT_ERR_SHAPE, "%s: logits are not aligned to their type", who);
  return ot_check_device(ctx, who);
}

}  // namespace
}  // namespace otv

using namespace otv;

#pragma GCC visibility push(default)
extern "C" {

int ot_token_logprobs(ot_ctx* ctx, const ot_logprob_in* in, ot_logprob_out* out) {
  if (!ctx || !in || !out) return ot_fail(OT_ERR_NULL, "ot_token_logprobs: ctx, in and out must not be NULL");
  if (const int bad = check_in(ctx, in, "ot_token_logprobs")) return bad;
  if (in->M == 0) return OT_OK;
  if ((in->n_tok > 0 && !out->logprob) || (in->n_top > 0 && (!out->top_ids || !out->top_logprobs)))
    return ot_fail(OT_ERR_NULL, "ot_token_logprobs: logprob, top_ids and top_logprobs are required where they have entries");
  if (!out->row_max != !out->row_sumexp) return ot_fail(OT_ERR_NULL, "ot_token_logprobs: row_max and row_sumexp come together");
  hipLaunchKernelGGL(logprob_kernel, dim3((unsigned)in->M), dim3(256), 0, ctx->stream, LogprobArgs{*in, *out});
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_token_logprobs: launch");
}

int ot_token_logprobs_grad(ot_ctx* ctx, const ot_logprob_in* in, const ot_logprob_out* fwd, const float* grad_logprob, const float* grad_entropy,
                           void* grad, int64_t ld_grad) {
  if (!ctx || !in || !fwd) return ot_fail(OT_ERR_NULL, "ot_token_logprobs_grad: ctx, in and forward must not be NULL");
  if (const int bad = check_in(ctx, in, "ot_token_logprobs_grad")) return bad;
  if (ld_grad < in->V) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: ld_grad = %lld is below V = %d", (long long)ld_grad, in->V);
  if (in->M == 0) return OT_OK;
  if (!grad || !fwd->row_max || !fwd->row_sumexp || (grad_entropy && !fwd->entropy))
    return ot_fail(OT_ERR_NULL, "ot_token_logprobs_grad: grad, row_max, row_sumexp and (with grad_entropy) entropy must not be NULL");
  if (reinterpret_cast<uintptr_t>(grad) % (in->dtype == OT_BF16 ? 2 : 4))
    return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: grad is not aligned to its type");
  if (grad == in->logits && ld_grad != in->ld) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: in place, ld_grad must be ld");
  const int chunks = ceil_div(in->V, kGradChunk);
  if ((int64_t)chunks * in->M > 0x7FFFFFFF) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: %d rows of %d ids are too many for a launch", in->M, in->V);
  const LogprobGradArgs a{*in, fwd->row_max, fwd->row_sumexp, fwd->entropy, grad_logprob, grad_entropy, grad, ld_grad};
  hipLaunchKernelGGL(logprob_grad_kernel, dim3((unsigned)(chunks * in->M)), dim3(256), 0, ctx->stream, a, chunks);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_token_logprobs_grad: launch");
}

}  // extern "C"
#pragma GCC visibility pop
