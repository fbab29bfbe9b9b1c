// C ABI of libmala.so: argument validation, workspace sizing and kernel launches.
// Declarations and the contract of every entry point are in include/mala.h.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <mutex>

#include "mala.h"
#include "mala_device.h"
#include "mala_kernels.h"
#include "mala_paged.h"
#include "mala_rope.h"
#include "mala_rows.h"

namespace {

thread_local char g_err[512] = "";

int fail(int status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return status;
}

int hip_fail(hipError_t e, const char* where) {
  snprintf(g_err, sizeof(g_err), "%s: %s", where, hipGetErrorString(e));
  return MALA_ERR_HIP;
}

size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Backward workspace: D_q = rowsum(O_q * dO_q) for every query row, then the dQ pass's
// tile decisions for the key-major pass (one byte per query tile, query head and
// 128-key block; query-tile rows as mask_rows gives them).
size_t dvec_bytes(long rows) { return round_up((size_t)rows * sizeof(float), 256); }
int mask_rows(bool packed, int B, int Nq) {
  return packed ? Nq / mala::kBq + B : B * ((Nq + mala::kBq - 1) / mala::kBq);
}
size_t mask_bytes(bool packed, int B, int Hq, int Nq, int max_k) {
  const size_t nkblk = (size_t)(max_k + mala::kBwdKeys - 1) / mala::kBwdKeys;
  return round_up((size_t)Hq * nkblk * mask_rows(packed, B, Nq), 256);
}
size_t part_bytes_packed(int num_seqs, int max_q, int total_k, int Hq, int Hkv, int D) {
  int psize, nparts;
  mala::dkdv_split_packed(num_seqs, max_q, total_k, Hq, Hkv, &psize, &nparts);
  return nparts > 1 ? round_up((size_t)nparts * 2 * Hkv * total_k * D * sizeof(float), 256) : 0;
}
// fp32 partial dV and dK of every part of the split sweeps (fixed-length batches)
size_t part_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int D) {
  int psize, nparts;
  mala::dkdv_split(B, Hq, Hkv, Nq, Nk, &psize, &nparts);
  return nparts > 1 ? round_up((size_t)nparts * 2 * B * Hkv * Nk * D * sizeof(float), 256) : 0;
}
size_t bwd_workspace(bool packed, int B, int Hq, int Hkv, int Nq, int max_k, int D) {
  const long rows = packed ? (long)Hq * Nq : (long)B * Hq * Nq;
  return dvec_bytes(rows) + mask_bytes(packed, B, Hq, Nq, max_k) +
         (packed ? 0 : part_bytes(B, Hq, Hkv, Nq, max_k, D));
}

int check_common(int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal, float scale, float tau) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0)
    return fail(MALA_ERR_INVALID_ARG, "non-positive size (B, Hq, Hkv, Nq, Nk)");
  if (Hq % Hkv != 0) return fail(MALA_ERR_INVALID_ARG, "Hq (%d) is not a multiple of Hkv (%d)", Hq, Hkv);
  if (Nq > Nk) return fail(MALA_ERR_INVALID_ARG, "Nq (%d) > Nk (%d)", Nq, Nk);
  if (!(tau >= 0.f) || isinf(tau)) return fail(MALA_ERR_INVALID_ARG, "tau must be finite and >= 0");
  if (!(scale > 0.f) || isinf(scale)) return fail(MALA_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (causal != 1) return fail(MALA_ERR_UNSUPPORTED, "only causal attention is supported");
  if (D != 64 && D != 128) return fail(MALA_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", D);
  return MALA_OK;
}

// The training kernels address one (batch, head) slice from a tile start through
// buffer resources whose range is a 32-bit byte count: Nk x D bf16 values must fit.
int check_slice_range(int Nk, int D) {
  const long long bytes = (long long)Nk * D * 2;
  if (bytes > 0xffffffffLL)
    return fail(MALA_ERR_UNSUPPORTED, "Nk x D x 2 = %lld bytes exceeds the 32-bit slice range", bytes);
  return MALA_OK;
}

float log2_tau(float tau) { return tau > 0.f ? log2f(tau) : -INFINITY; }

}  // namespace

extern "C" {

mala_geometry_t mala_geometry(int head_dim, int pass) {
  mala_geometry_t g = {0, 0};
  if (head_dim != 64 && head_dim != 128) return g;
  if (pass == MALA_PASS_FWD || pass == MALA_PASS_BWD) {
    g.block_q = mala::kBq;
    g.block_k = mala::kBk;
  } else if (pass == MALA_PASS_DECODE) {
    g.block_q = 1;
    g.block_k = mala::kDecBk;
  }
  return g;
}

const char* mala_strerror(int status) {
  switch (status) {
    case MALA_OK: return "success";
    case MALA_ERR_INVALID_ARG: return "invalid argument";
    case MALA_ERR_UNSUPPORTED: return "unsupported configuration";
    case MALA_ERR_WORKSPACE: return "workspace missing or too small";
    case MALA_ERR_HIP: return "HIP runtime error";
    default: return "unknown status";
  }
}

const char* mala_last_error(void) { return g_err; }

}  // extern "C"

namespace {

// Packed batches: the query-row / key-row starts of the sequences (cu null for the
// fixed-length layout, cu_k null for the same starts as cu) and their longest
// lengths.
struct Packed {
  const int32_t* cu;
  const int32_t* cu_k;
  int max_q, max_k;
};

// Shared by the fixed-length and packed entry points: B slices (sequences) of
// Nq / Nk rows each (packed: Nq, Nk = the query / key totals, the head strides).
int run_fwd(const void* q, const void* k, const void* v, const Packed& pk,
            void* o, int o_dtype, float* lse, int32_t* row_tiles, int64_t* counters, int B,
            int Hq, int Hkv, int Nq, int Nk, int D, float scale, float tau, hipStream_t s) {
  if (counters) {
    hipError_t e = mala::launch_fill_zero(counters, mala::kNumCounters * sizeof(int64_t), s);
    if (e != hipSuccess) return hip_fail(e, "mala_fwd: clearing counters");
  }
  mala::FwdParams p;
  p.q = (const __bf16*)q;
  p.k = (const __bf16*)k;
  p.v = (const __bf16*)v;
  p.o = o;
  p.o_bf16 = o_dtype == MALA_OUT_BF16;
  p.lse = lse;
  p.row_tiles = row_tiles;
  p.counters = (unsigned long long*)counters;
  p.cu = pk.cu;
  p.cu_k = pk.cu_k;
  p.max_len = pk.cu ? pk.max_q : Nq;
  p.max_len_k = pk.cu ? pk.max_k : Nk;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Nq = Nq; p.Nk = Nk;
  p.scale2 = scale * mala::kLog2e;
  p.log2tau = log2_tau(tau);
  p.nqblk = (p.max_len + mala::kFwdRows - 1) / mala::kFwdRows;
  hipError_t e = mala::launch_fwd(p, D, s);
  if (e != hipSuccess) return hip_fail(e, "mala_fwd: kernel launch");
  return MALA_OK;
}

int run_bwd(const void* q, const void* k, const void* v, const Packed& pk,
            const void* o, int o_dtype, const float* lse, const void* dout, void* dq, void* dk,
            void* dv, int grad_dtype, int32_t* row_tiles, int64_t* counters, void* workspace,
            size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int D, float scale, float tau,
            hipStream_t s) {
  hipError_t e;
  // D_q over every row of the q-shaped tensors (packed: all heads x total rows)
  const long rows = pk.cu ? (long)Hq * Nq : (long)B * Hq * Nq;
  if (counters && (e = mala::launch_fill_zero(counters, mala::kNumCounters * sizeof(int64_t), s)) != hipSuccess)
    return hip_fail(e, "mala_bwd: clearing counters");
  float* dvec = (float*)workspace;
  mala::BwdParams p;
  p.q = (const __bf16*)q;
  p.k = (const __bf16*)k;
  p.v = (const __bf16*)v;
  p.dout = (const __bf16*)dout;
  p.lse = lse;
  p.o = o;
  p.o_bf16 = o_dtype == MALA_OUT_BF16;
  p.dvec = dvec;
  p.dq = dq; p.dk = dk; p.dv = dv;
  p.grad_bf16 = grad_dtype == MALA_OUT_BF16;
  p.row_tiles = row_tiles;
  p.counters = (unsigned long long*)counters;
  p.cu = pk.cu;
  p.cu_k = pk.cu_k;
  p.max_len = pk.cu ? pk.max_q : Nq;
  p.max_len_k = pk.cu ? pk.max_k : Nk;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Nq = Nq; p.Nk = Nk;
  p.scale = scale;
  p.scale2 = scale * mala::kLog2e;
  p.log2tau = log2_tau(tau);
  p.nkblk = (p.max_len_k + mala::kBwdKeys - 1) / mala::kBwdKeys;
  p.nqblk = (p.max_len + mala::kDqRows - 1) / mala::kDqRows;
  p.mask = (uint8_t*)workspace + dvec_bytes(rows);
  p.mask_rows = mask_rows(pk.cu != nullptr, B, Nq);
  const size_t before = dvec_bytes(rows) + mask_bytes(pk.cu != nullptr, B, Hq, Nq, p.max_len_k);
  p.part = (float*)((char*)workspace + before);
  p.part_rows = (pk.cu ? 1 : (size_t)B) * Hkv * Nk;
  if (!pk.cu) {
    mala::dkdv_split(B, Hq, Hkv, Nq, Nk, &p.psize, &p.nparts);
  } else {
    // a workspace without room for the parts (e.g. sized for fewer keys) gives whole sweeps
    mala::dkdv_split_packed(B, pk.max_q, Nk, Hq, Hkv, &p.psize, &p.nparts);
    if (workspace_bytes < before + part_bytes_packed(B, pk.max_q, Nk, Hq, Hkv, D)) {
      p.psize = 1 << 30;
      p.nparts = 1;
    }
  }
  if ((e = mala::launch_bwd(p, D, s)) != hipSuccess) return hip_fail(e, "mala_bwd: kernel launch");
  return MALA_OK;
}

int check_dtype(int d, const char* what) {
  if (d != MALA_OUT_F32 && d != MALA_OUT_BF16)
    return fail(MALA_ERR_INVALID_ARG, "%s must be MALA_OUT_F32 or MALA_OUT_BF16, got %d", what, d);
  return MALA_OK;
}

int check_varlen(const int32_t* cu_q, const int32_t* cu_k, int num_seqs, int max_q, int max_k,
                 int total_q, int total_k, int Hq, int Hkv, int D, float scale, float tau) {
  if (!cu_q) return fail(MALA_ERR_INVALID_ARG, "null cu_seqlens_q");
  if (num_seqs <= 0 || max_q <= 0 || max_k <= 0 || total_q <= 0 || total_k <= 0)
    return fail(MALA_ERR_INVALID_ARG, "non-positive size (num_seqs, max_seqlen, total)");
  if (max_q > total_q || max_k > total_k)
    return fail(MALA_ERR_INVALID_ARG, "max_seqlen above its total (%d > %d or %d > %d)", max_q,
                total_q, max_k, total_k);
  if (!cu_k && (total_k != total_q || max_k != max_q))
    return fail(MALA_ERR_INVALID_ARG, "without cu_seqlens_k the key totals must equal the query's");
  int st = check_common(1, Hq, Hkv, total_q, total_k, D, 1, scale, tau);
  if (!st) st = check_slice_range(total_k, D);
  return st;
}

int check_decode(const void* q, const void* k_cache, const void* v_cache, const void* o,
                 const float* lse, int num_splits, int B, int Hq, int Hkv, int Nk, int D,
                 float scale, float tau, int out_dtype) {
  if (!q || !k_cache || !v_cache || !o || !lse)
    return fail(MALA_ERR_INVALID_ARG, "null q, k_cache, v_cache, o or lse");
  int st = check_common(B, Hq, Hkv, 1, Nk, D, 1, scale, tau);
  if (!st) st = check_dtype(out_dtype, "out_dtype");
  if (st) return st;
  if (num_splits < 1) return fail(MALA_ERR_INVALID_ARG, "num_splits must be >= 1");
  return MALA_OK;
}

// The split kernel writes every partial [B, Hq, num_splits, D + 4] (also for splits
// without tiles: o = 0, lse = -inf) before the merge kernel reads it, so the buffer
// needs no clearing; with one split it writes the outputs themselves.
int run_decode(const void* q, const void* k_cache, const void* v_cache, const int32_t* cache_lens,
               void* o, float* lse, int32_t* head_tiles, int64_t* counters, int num_splits,
               float* part, int B, int Hq, int Hkv, int Nk, int D, float scale, float tau,
               int out_dtype, hipStream_t s) {
  hipError_t e;
  if (counters &&
      (e = mala::launch_fill_zero(counters, mala::kNumCounters * sizeof(int64_t), s)) != hipSuccess)
    return hip_fail(e, "mala_decode: clearing counters");
  const int T = (Nk + mala::kDecBk - 1) / mala::kDecBk;
  mala::DecParams p;
  p.q = (const __bf16*)q;
  p.k = (const __bf16*)k_cache;
  p.v = (const __bf16*)v_cache;
  p.lens = cache_lens;
  p.part = part;
  p.counters = (unsigned long long*)counters;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Nk = Nk;
  p.S = num_splits;
  p.nchunk = (Hq / Hkv + 15) / 16;
  p.T = T;
  p.tps = (T + num_splits - 1) / num_splits;
  p.scale2 = scale * mala::kLog2e;
  p.thr2 = log2_tau(tau) - log2f((float)Nk);
  p.log2tau = log2_tau(tau);
  p.o = o;
  p.o_bf16 = out_dtype == MALA_OUT_BF16;
  p.lse = lse;
  p.head_tiles = head_tiles;
  if ((e = mala::launch_decode(p, D, s)) != hipSuccess) return hip_fail(e, "mala_decode: kernel launch");
  return MALA_OK;
}

// The decode buffer of mala_decode_noalloc: a file-scope device array that every GPU
// the library runs on holds until the process ends.  In host code `scratch` names a
// host-side stand-in, not the array's device address: the address on a device comes
// from hipGetSymbolAddress, looked up once per device (with that device current) and
// kept in g_scratch; only that address is passed to kernels.
constexpr size_t kDecodeScratchBytes = MALA_DECODE_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[kDecodeScratchBytes];
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch[kMaxDevices];

// The device address of `scratch` on the device of stream s (the current device for
// the null stream).
int scratch_address(hipStream_t s, void** out) {
  int dev = 0;
  hipError_t e = s ? hipStreamGetDevice(s, &dev) : hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "mala_decode_noalloc: device of the stream");
  if (dev < 0 || dev >= kMaxDevices)
    return fail(MALA_ERR_UNSUPPORTED, "mala_decode_noalloc: device %d beyond %d", dev, kMaxDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch[dev]) {
    int cur = 0;
    if ((e = hipGetDevice(&cur)) != hipSuccess) return hip_fail(e, "mala_decode_noalloc: hipGetDevice");
    if (cur != dev && (e = hipSetDevice(dev)) != hipSuccess)
      return hip_fail(e, "mala_decode_noalloc: hipSetDevice");
    void* ptr = nullptr;
    const hipError_t eg = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (cur != dev && (e = hipSetDevice(cur)) != hipSuccess)
      return hip_fail(e, "mala_decode_noalloc: restoring the current device");
    if (eg != hipSuccess) return hip_fail(eg, "mala_decode_noalloc: hipGetSymbolAddress");
    if (!ptr) return fail(MALA_ERR_HIP, "mala_decode_noalloc: no device address for the buffer");
    g_scratch[dev] = ptr;
  }
  *out = g_scratch[dev];
  return MALA_OK;
}

}  // namespace

extern "C" {

int mala_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t* row_tiles,
             int64_t* counters, int B, int Hq, int Hkv, int Nq, int Nk, int D, int causal,
             float scale, float tau, int out_dtype, void* stream) {
  g_err[0] = 0;
  if (!q || !k || !v || !o || !lse) return fail(MALA_ERR_INVALID_ARG, "null q, k, v, o or lse");
  int st = check_common(B, Hq, Hkv, Nq, Nk, D, causal, scale, tau);
  if (!st) st = check_slice_range(Nk, D);
  if (!st) st = check_dtype(out_dtype, "out_dtype");
  if (st) return st;
  return run_fwd(q, k, v, Packed{}, o, out_dtype, lse, row_tiles, counters, B, Hq, Hkv, Nq, Nk,
                 D, scale, tau, (hipStream_t)stream);
}

int mala_fwd_varlen(const void* q, const void* k, const void* v, const int32_t* cu_seqlens_q,
                    const int32_t* cu_seqlens_k, void* o, float* lse, int32_t* row_tiles,
                    int64_t* counters, int num_seqs, int max_seqlen_q, int max_seqlen_k,
                    int total_q, int total_k, int Hq, int Hkv, int D, float scale, float tau,
                    int out_dtype, void* stream) {
  g_err[0] = 0;
  if (!q || !k || !v || !o || !lse) return fail(MALA_ERR_INVALID_ARG, "null q, k, v, o or lse");
  int st = check_varlen(cu_seqlens_q, cu_seqlens_k, num_seqs, max_seqlen_q, max_seqlen_k,
                        total_q, total_k, Hq, Hkv, D, scale, tau);
  if (!st) st = check_dtype(out_dtype, "out_dtype");
  if (st) return st;
  return run_fwd(q, k, v, Packed{cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k}, o,
                 out_dtype, lse, row_tiles, counters, num_seqs, Hq, Hkv, total_q, total_k, D,
                 scale, tau, (hipStream_t)stream);
}

size_t mala_bwd_workspace_size(int B, int Hq, int Hkv, int Nq, int Nk, int D) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0 || Hq % Hkv || Nq > Nk ||
      (D != 64 && D != 128))
    return 0;
  return bwd_workspace(false, B, Hq, Hkv, Nq, Nk, D);
}

size_t mala_bwd_varlen_workspace_size(int num_seqs, int max_seqlen_k, int total_q, int Hq,
                                      int Hkv, int D) {
  if (num_seqs <= 0 || max_seqlen_k <= 0 || total_q <= 0 || Hq <= 0 || Hkv <= 0) return 0;
  // with the parts of self-attention (keys = queries)
  return bwd_workspace(true, num_seqs, Hq, Hkv, total_q, max_seqlen_k, D) +
         (Hq % Hkv ? 0 : part_bytes_packed(num_seqs, max_seqlen_k, total_q, Hq, Hkv, D));
}

int mala_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
             const void* dout, void* dq, void* dk, void* dv, int32_t* row_tiles,
             int64_t* counters, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
             int Nq, int Nk, int D, int causal, float scale, float tau, int o_dtype,
             int grad_dtype, void* stream) {
  g_err[0] = 0;
  if (!q || !k || !v || !o || !lse || !dout || !dq || !dk || !dv)
    return fail(MALA_ERR_INVALID_ARG, "null tensor argument");
  int st = check_common(B, Hq, Hkv, Nq, Nk, D, causal, scale, tau);
  if (!st) st = check_slice_range(Nk, D);
  if (!st) st = check_dtype(o_dtype, "o_dtype");
  if (!st) st = check_dtype(grad_dtype, "grad_dtype");
  if (st) return st;
  const size_t need = mala_bwd_workspace_size(B, Hq, Hkv, Nq, Nk, D);
  if (!workspace || workspace_bytes < need)
    return fail(MALA_ERR_WORKSPACE, "mala_bwd needs %zu workspace bytes, got %zu", need, workspace_bytes);
  if (((uintptr_t)workspace) % 16) return fail(MALA_ERR_WORKSPACE, "workspace not 16-byte aligned");
  return run_bwd(q, k, v, Packed{}, o, o_dtype, lse, dout, dq, dk, dv, grad_dtype, row_tiles,
                 counters, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, D, scale, tau,
                 (hipStream_t)stream);
}

int mala_bwd_varlen(const void* q, const void* k, const void* v, const int32_t* cu_seqlens_q,
                    const int32_t* cu_seqlens_k, const void* o, const float* lse,
                    const void* dout, void* dq, void* dk, void* dv, int32_t* row_tiles,
                    int64_t* counters, void* workspace, size_t workspace_bytes, int num_seqs,
                    int max_seqlen_q, int max_seqlen_k, int total_q, int total_k, int Hq,
                    int Hkv, int D, float scale, float tau, int o_dtype, int grad_dtype,
                    void* stream) {
  g_err[0] = 0;
  if (!q || !k || !v || !o || !lse || !dout || !dq || !dk || !dv)
    return fail(MALA_ERR_INVALID_ARG, "null tensor argument");
  int st = check_varlen(cu_seqlens_q, cu_seqlens_k, num_seqs, max_seqlen_q, max_seqlen_k,
                        total_q, total_k, Hq, Hkv, D, scale, tau);
  if (!st) st = check_dtype(o_dtype, "o_dtype");
  if (!st) st = check_dtype(grad_dtype, "grad_dtype");
  if (st) return st;
  const size_t need = bwd_workspace(true, num_seqs, Hq, Hkv, total_q, max_seqlen_k, D);
  if (!workspace || workspace_bytes < need)
    return fail(MALA_ERR_WORKSPACE, "mala_bwd_varlen needs %zu workspace bytes, got %zu", need,
                workspace_bytes);
  if (((uintptr_t)workspace) % 16) return fail(MALA_ERR_WORKSPACE, "workspace not 16-byte aligned");
  return run_bwd(q, k, v, Packed{cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k}, o,
                 o_dtype, lse, dout, dq, dk, dv, grad_dtype, row_tiles, counters, workspace,
                 workspace_bytes, num_seqs, Hq, Hkv, total_q, total_k, D, scale, tau, (hipStream_t)stream);
}

size_t mala_decode_workspace_size(int B, int Hq, int D, int num_splits) {
  if (B <= 0 || Hq <= 0 || num_splits <= 0 || (D != 64 && D != 128)) return 0;
  return round_up((size_t)B * Hq * num_splits * (D + mala::kDecStride) * sizeof(float), 256);
}

int mala_decode(const void* q, const void* k_cache, const void* v_cache,
                const int32_t* cache_lens, void* o, float* lse, int32_t* head_tiles,
                int64_t* counters, int num_splits, void* workspace, size_t workspace_bytes,
                int B, int Hq, int Hkv, int Nk, int D, float scale, float tau, int out_dtype,
                void* stream) {
  g_err[0] = 0;
  int st = check_decode(q, k_cache, v_cache, o, lse, num_splits, B, Hq, Hkv, Nk, D, scale, tau,
                        out_dtype);
  if (st) return st;
  const size_t need = mala_decode_workspace_size(B, Hq, D, num_splits);
  if (!workspace || workspace_bytes < need)
    return fail(MALA_ERR_WORKSPACE, "mala_decode needs %zu workspace bytes, got %zu", need,
                workspace_bytes);
  if (((uintptr_t)workspace) % 16) return fail(MALA_ERR_WORKSPACE, "workspace not 16-byte aligned");
  return run_decode(q, k_cache, v_cache, cache_lens, o, lse, head_tiles, counters, num_splits,
                    (float*)workspace, B, Hq, Hkv, Nk, D, scale, tau, out_dtype,
                    (hipStream_t)stream);
}

int mala_decode_noalloc(const void* q, const void* k_cache, const void* v_cache,
                        const int32_t* cache_lens, void* o, float* lse, int32_t* head_tiles,
                        int64_t* counters, int num_splits, int B, int Hq, int Hkv, int Nk, int D,
                        float scale, float tau, int out_dtype, void* stream) {
  g_err[0] = 0;
  int st = check_decode(q, k_cache, v_cache, o, lse, num_splits, B, Hq, Hkv, Nk, D, scale, tau,
                        out_dtype);
  if (st) return st;
  const size_t need = mala_decode_workspace_size(B, Hq, D, num_splits);
  if (need > kDecodeScratchBytes)
    return fail(MALA_ERR_WORKSPACE,
                "mala_decode_noalloc: the split partials need %zu bytes, more than the library's "
                "%zu-byte decode buffer (use mala_decode with a workspace, or fewer splits)",
                need, kDecodeScratchBytes);
  void* part = nullptr;
  hipStream_t s = (hipStream_t)stream;
  if ((st = scratch_address(s, &part)) != MALA_OK) return st;
  return run_decode(q, k_cache, v_cache, cache_lens, o, lse, head_tiles, counters, num_splits,
                    (float*)part, B, Hq, Hkv, Nk, D, scale, tau, out_dtype, s);
}

}  // extern "C"

// ---------------------------------------------------------------- paged KV cache
namespace {

// Checks a cache and fills its kernel form.
int check_cache(const mala_paged_cache_t* c, mala::PagedCache* out) {
  if (!c || !c->k_pages || !c->v_pages)
    return fail(MALA_ERR_INVALID_ARG, "null cache, k_pages or v_pages");
  if (c->num_pages <= 0 || c->page_size <= 0 || c->Hkv <= 0)
    return fail(MALA_ERR_INVALID_ARG, "non-positive size (num_pages, page_size, Hkv)");
  if (c->dtype != MALA_CACHE_BF16 && c->dtype != MALA_CACHE_E4M3 && c->dtype != MALA_CACHE_E4M3_BLOCK)
    return fail(MALA_ERR_INVALID_ARG, "cache dtype must be a MALA_CACHE_*, got %d", c->dtype);
  if (c->dtype != MALA_CACHE_E4M3 && (c->k_scale || c->v_scale))
    return fail(MALA_ERR_INVALID_ARG, "only a MALA_CACHE_E4M3 has scales per head");
  // (the block scales are behind the fields that a bf16 or e4m3 cache has to give)
  const bool block = c->dtype == MALA_CACHE_E4M3_BLOCK;
  if (block && (!c->k_block_scale || !c->v_block_scale))
    return fail(MALA_ERR_INVALID_ARG, "null k_block_scale or v_block_scale");
  if (c->D != 64 && c->D != 128)
    return fail(MALA_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", c->D);
  if (c->page_size % mala::kPageRows)
    return fail(MALA_ERR_UNSUPPORTED, "page_size %d is not a multiple of %d", c->page_size, mala::kPageRows);
  if ((int64_t)c->num_pages * c->page_size > INT32_MAX)
    return fail(MALA_ERR_UNSUPPORTED, "num_pages x page_size reaches 2^31");
  const int64_t size = c->dtype == MALA_CACHE_BF16 ? 2 : 1;
  const int64_t per_16 = 16 / size;       // elements
  for (int64_t s : {c->page_stride, c->head_stride, c->token_stride})
    if (s < c->D || s % per_16)
      return fail(MALA_ERR_INVALID_ARG, "cache strides must be at least D and multiples of 16 bytes");
  // (compared by division: products of strides as given can pass 64 bits.  Every axis below 2^60
  // bytes, so that the kernels' sums of them fit too.)
  constexpr int64_t kMost = (int64_t)1 << 60;
  if (c->page_stride > kMost / size / c->num_pages || c->head_stride > kMost / size / c->Hkv)
    return fail(MALA_ERR_UNSUPPORTED, "cache stride too large");
  if (c->token_stride > INT32_MAX / (size * mala::kPageRows))
    return fail(MALA_ERR_UNSUPPORTED, "16 rows of the cache span 2^31 bytes");
  if ((uintptr_t)c->k_pages % 16 || (uintptr_t)c->v_pages % 16)
    return fail(MALA_ERR_INVALID_ARG, "k_pages or v_pages not 16-byte aligned");
  if (block) {
    const uintptr_t a = (uintptr_t)c->k_block_scale, b = (uintptr_t)c->v_block_scale;
    const uintptr_t n = (uintptr_t)c->num_pages * c->Hkv * (c->page_size / mala::kPageRows);
    if (a < b + n && b < a + n)
      return fail(MALA_ERR_INVALID_ARG, "k_block_scale and v_block_scale share memory");
  }
  if (out) {
    out->k = (char*)c->k_pages;
    out->v = (char*)c->v_pages;
    out->ks = c->k_scale;
    out->vs = c->v_scale;
    out->page_stride = c->page_stride * size;
    out->head_stride = c->head_stride * size;
    out->token_stride = c->token_stride * size;
    out->num_pages = c->num_pages;
    out->page_size = c->page_size;
    out->Hkv = c->Hkv;
    out->kb = block ? c->k_block_scale : nullptr;
    out->vb = block ? c->v_block_scale : nullptr;
    out->fmt = block ? mala::kCacheBlock : c->dtype == MALA_CACHE_E4M3 ? mala::kCacheE4M3 : mala::kCacheBf16;
  }
  return MALA_OK;
}

// A write's block scales lie in no row of the pages: others would be rows and scales at once.
int check_scales_apart(const mala::PagedCache& c, int D) {
  if (c.fmt != mala::kCacheBlock) return MALA_OK;
  const mala::Rows pages = {(uintptr_t)c.k, D, {c.page_stride, c.head_stride, c.token_stride},
                            {c.num_pages, c.Hkv, c.page_size}};
  for (const char* rows : {c.k, c.v})
    for (const uint8_t* scales : {c.kb, c.vb}) {
      const mala::Rows x = {(uintptr_t)scales, (int64_t)c.num_pages * c.Hkv * (c.page_size / mala::kPageRows),
                            {0, 0, 0}, {1, 1, 1}};
      mala::Rows y = pages;
      y.base = (uintptr_t)rows;
      const mala::Shared shared = mala::rows_meet(x, y);
      if (shared == mala::kShare) return fail(MALA_ERR_INVALID_ARG, "block scales share memory with the pages");
      if (shared) return fail(MALA_ERR_UNSUPPORTED, "block scales and pages cannot be told apart");
    }
  return MALA_OK;
}

// The arguments of a write, and its kernel form (nothing past the cache where there is no token).
int check_write(const void* k_new, const void* v_new, int64_t new_token_stride, int64_t new_head_stride,
                const int32_t* slots, const mala_paged_cache_t* cache, int num_tokens,
                mala::PagedWriteParams* p) {
  const int st = check_cache(cache, &p->c);
  if (st) return st;
  if (num_tokens < 0) return fail(MALA_ERR_INVALID_ARG, "negative num_tokens");
  if (!num_tokens) return MALA_OK;
  if (!k_new || !v_new || !slots) return fail(MALA_ERR_INVALID_ARG, "null k_new, v_new or slots");
  if ((uintptr_t)k_new % 16 || (uintptr_t)v_new % 16 || new_token_stride % 8 || new_head_stride % 8 ||
      new_token_stride < 0 || new_head_stride < 0)
    return fail(MALA_ERR_INVALID_ARG, "rows of k_new and v_new must be 16-byte aligned");
  if (new_token_stride > INT64_MAX / 8 / num_tokens || new_head_stride > INT64_MAX / 8 / cache->Hkv)
    return fail(MALA_ERR_UNSUPPORTED, "k_new stride too large");
  // (a thread per 16 bytes of a row of the cache; of blocks, as the launch rule says)
  const int64_t threads = p->c.fmt == mala::kCacheBlock
                              ? 256 * mala::block_write_plan(num_tokens, cache->Hkv, false).groups
                              : (int64_t)num_tokens * (cache->D / (p->c.fmt == mala::kCacheBf16 ? 8 : 16));
  if (threads > UINT32_MAX - 255)
    return fail(MALA_ERR_UNSUPPORTED, "a launch of 2^32 threads or more (num_tokens %d)", num_tokens);
  p->k = (const char*)k_new;
  p->v = (const char*)v_new;
  p->token_stride = new_token_stride * 2;
  p->head_stride = new_head_stride * 2;
  p->slots = slots;
  p->T = num_tokens;
  p->chunk = p->units = 0;
  return MALA_OK;
}

// ---------------------------------------------------------------- rotary positions
// Rows that a launch reads or writes in any order beside those that it writes.
int check_apart(const mala::Rows& written, const char* name, const mala::Rows& other, const char* what) {
  const mala::Shared shared = mala::rows_meet(written, other);
  if (shared == mala::kShare)
    return fail(MALA_ERR_INVALID_ARG, "the output of %s shares memory with %s", name, what);
  if (shared) return fail(MALA_ERR_UNSUPPORTED, "the output of %s and %s cannot be told apart", name, what);
  return MALA_OK;
}

// One tensor's rows, B x heads x T of them (all above 0).
struct TurnedRows {
  mala::Rows x, out;
};
int check_rows(const mala_rope_rows_t* r, const char* name, int B, int T, int D, int in_size, int out_size,
               mala::RopeRows* out, TurnedRows* rows) {
  if (!r->x || !r->out) return fail(MALA_ERR_INVALID_ARG, "null x or out of %s", name);
  if (r->heads <= 0) return fail(MALA_ERR_INVALID_ARG, "non-positive heads of %s", name);
  if (r->heads > 65535) return fail(MALA_ERR_UNSUPPORTED, "%d heads of %s", r->heads, name);
  if ((uintptr_t)r->x % 16 || (uintptr_t)r->out % 16)
    return fail(MALA_ERR_INVALID_ARG, "x or out of %s not 16-byte aligned", name);
  const int64_t n[3] = {B, r->heads, T};
  int64_t in[3] = {r->x_batch_stride, r->x_head_stride, r->x_token_stride};
  int64_t to[3] = {r->out_batch_stride, r->out_head_stride, r->out_token_stride};
  int64_t in_b[3], to_b[3];
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) in[i] = to[i] = 0;
    if (in[i] < 0 || to[i] < 0 || in[i] % (16 / in_size) || to[i] % (16 / out_size))
      return fail(MALA_ERR_INVALID_ARG, "strides of %s must be multiples of 16 bytes, not negative", name);
    // every axis below 2^60 bytes (compared by division)
    constexpr int64_t kMost = (int64_t)1 << 60;
    if (in[i] > kMost / in_size / n[i] || to[i] > kMost / out_size / n[i])
      return fail(MALA_ERR_UNSUPPORTED, "stride of %s too large", name);
    in_b[i] = in[i] * in_size;
    to_b[i] = to[i] * out_size;
  }
  // rows of an output that share memory would be written by several threads
  const mala::Rows x = {(uintptr_t)r->x, (int64_t)D * in_size, {in_b[0], in_b[1], in_b[2]}, {n[0], n[1], n[2]}};
  const mala::Rows y = {(uintptr_t)r->out, (int64_t)D * out_size, {to_b[0], to_b[1], to_b[2]}, {n[0], n[1], n[2]}};
  const mala::Shared shared = mala::rows_overlap(y);
  if (shared == mala::kShare) return fail(MALA_ERR_INVALID_ARG, "rows of the output of %s overlap", name);
  if (shared) return fail(MALA_ERR_UNSUPPORTED, "the rows of the output of %s cannot be told apart", name);
  bool same = r->x == r->out && in_size == out_size;
  for (int i = 0; i < 3; ++i) same = same && in[i] == to[i];
  if (!same && x.base < y.base + y.extent() && y.base < x.base + x.extent())
    return fail(MALA_ERR_INVALID_ARG, "the output of %s meets its input without being it", name);
  *rows = {x, y};
  *out = {(const char*)r->x, (char*)r->out, in_b[0], in_b[1], in_b[2], to_b[0], to_b[1], to_b[2], r->heads};
  return MALA_OK;
}

int check_turn(const mala_rope_t* rope, int B, int T, int D, int inverse, mala::Turn* out) {
  if (!rope || !rope->inv_freq) return fail(MALA_ERR_INVALID_ARG, "null rope or inv_freq");
  if (D != 64 && D != 128) return fail(MALA_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", D);
  if (rope->layout != MALA_ROPE_HALF && rope->layout != MALA_ROPE_INTERLEAVED)
    return fail(MALA_ERR_INVALID_ARG, "layout must be a MALA_ROPE_*, got %d", rope->layout);
  if (rope->rotary_dim <= 0 || rope->rotary_dim > D)
    return fail(MALA_ERR_INVALID_ARG, "rotary_dim %d not in 1 .. %d", rope->rotary_dim, D);
  if (rope->rotary_dim % 16) return fail(MALA_ERR_UNSUPPORTED, "rotary_dim %d is not a multiple of 16", rope->rotary_dim);
  if (!isfinite(rope->scale)) return fail(MALA_ERR_INVALID_ARG, "scale of the rotation must be finite");
  if ((uintptr_t)rope->inv_freq % 8 || (uintptr_t)rope->positions % 4)
    return fail(MALA_ERR_INVALID_ARG, "inv_freq or positions misaligned");
  if (rope->positions_batch_stride < 0)
    return fail(MALA_ERR_INVALID_ARG, "negative positions_batch_stride");
  if (rope->positions_batch_stride > ((int64_t)1 << 58) / std::max(B, 1))
    return fail(MALA_ERR_UNSUPPORTED, "positions_batch_stride too large");
  // (D / 16 threads per row)
  if ((int64_t)B * T > (UINT32_MAX - 255) / (D / 16))
    return fail(MALA_ERR_UNSUPPORTED, "a launch of 2^32 threads or more (%d x %d tokens)", B, T);
  *out = {rope->positions, rope->positions_batch_stride, rope->inv_freq, rope->rotary_dim,
          rope->layout == MALA_ROPE_INTERLEAVED, rope->scale, inverse ? -rope->scale : rope->scale};
  return MALA_OK;
}

// Decode workspace: where every sequence's partials lie, then the partials.
size_t paged_plan_bytes(int B) { return round_up((size_t)B * sizeof(int2), 256); }

int check_split_tokens(int split_tokens) {
  if (split_tokens <= 0 || split_tokens % mala::kDecBk)
    return fail(MALA_ERR_INVALID_ARG, "split_tokens %d is not a positive multiple of %d", split_tokens, mala::kDecBk);
  return MALA_OK;
}

}  // namespace

extern "C" {

int mala_paged_update(const int32_t* lens, const int32_t* new_lens, int32_t* block_table,
                      int32_t* free_ring, const int32_t* free_state, int32_t* lens_out,
                      int32_t* cu_seqlens, int32_t* slots, int32_t* positions,
                      int32_t* free_state_out, int num_seqs, int max_pages, int page_size,
                      int num_pages, int ring_size, int max_tokens, void* stream) {
  g_err[0] = 0;
  if (!lens || !new_lens || !block_table || !free_ring || !free_state || !lens_out || !cu_seqlens ||
      !free_state_out || (!slots && max_tokens))
    return fail(MALA_ERR_INVALID_ARG, "null argument");
  if (num_seqs <= 0 || max_pages <= 0 || page_size <= 0 || num_pages <= 0 || ring_size <= 0 || max_tokens < 0)
    return fail(MALA_ERR_INVALID_ARG, "non-positive size");
  if (page_size % mala::kPageRows)
    return fail(MALA_ERR_UNSUPPORTED, "page_size %d is not a multiple of %d", page_size, mala::kPageRows);
  if ((double)num_seqs * max_pages * page_size > INT32_MAX || (int64_t)num_pages * page_size > INT32_MAX)
    return fail(MALA_ERR_UNSUPPORTED, "num_seqs x max_pages x page_size or num_pages x page_size reaches 2^31");
  // block_table and free_ring are inputs and outputs; an output shares no byte with any other array
  const struct {
    const int32_t* p;
    int64_t n;
  } arrays[] = {{lens, num_seqs}, {new_lens, num_seqs}, {free_state, 2},
                {block_table, (int64_t)num_seqs * max_pages}, {free_ring, ring_size},
                {lens_out, num_seqs}, {cu_seqlens, (int64_t)num_seqs + 1}, {slots, max_tokens},
                {positions, max_tokens}, {free_state_out, 4}};
  constexpr int kArrays = 10, kFirstOutput = 3;
  for (int j = kFirstOutput; j < kArrays; ++j)
    for (int i = 0; i < j; ++i) {
      const uintptr_t a = (uintptr_t)arrays[i].p, b = (uintptr_t)arrays[j].p;
      if (a && b && arrays[i].n && arrays[j].n && a < b + 4 * arrays[j].n && b < a + 4 * arrays[i].n)
        return fail(MALA_ERR_INVALID_ARG, "an output shares its memory with another argument");
    }
  const mala::PagedUpdateParams p = {lens, new_lens, block_table, free_ring, free_state, lens_out,
                                     cu_seqlens, slots, positions, free_state_out, num_seqs,
                                     max_pages, page_size, num_pages, ring_size, max_tokens};
  const hipError_t e = mala::launch_paged_update(p, (hipStream_t)stream);
  return e == hipSuccess ? MALA_OK : hip_fail(e, "mala_paged_update: kernel launch");
}

int mala_paged_write(const void* k_new, const void* v_new, int64_t new_token_stride,
                     int64_t new_head_stride, const int32_t* slots,
                     const mala_paged_cache_t* cache, int num_tokens, void* stream) {
  g_err[0] = 0;
  mala::PagedWriteParams p;
  int st = check_write(k_new, v_new, new_token_stride, new_head_stride, slots, cache, num_tokens, &p);
  if (st || !num_tokens) return st;
  if ((st = check_scales_apart(p.c, cache->D))) return st;
  const hipError_t e = mala::launch_paged_write(p, cache->D, (hipStream_t)stream);
  return e == hipSuccess ? MALA_OK : hip_fail(e, "mala_paged_write: kernel launch");
}

int mala_rope(const mala_rope_rows_t* q, const mala_rope_rows_t* k, const mala_rope_t* rope, int B, int T,
              int D, int in_dtype, int out_dtype, int inverse, void* stream) {
  g_err[0] = 0;
  if (!q) return fail(MALA_ERR_INVALID_ARG, "null q");
  if (B < 0 || T < 0) return fail(MALA_ERR_INVALID_ARG, "negative size (B, T)");
  mala::RopeParams p = {};
  int st = check_turn(rope, B, T, D, inverse, &p.turn);
  if (!st) st = check_dtype(in_dtype, "in_dtype");
  if (!st) st = check_dtype(out_dtype, "out_dtype");
  if (st || !B || !T) return st;
  const int in_size = in_dtype == MALA_OUT_BF16 ? 2 : 4, out_size = out_dtype == MALA_OUT_BF16 ? 2 : 4;
  TurnedRows qr, kr;
  if ((st = check_rows(q, "q", B, T, D, in_size, out_size, &p.r[0], &qr))) return st;
  if (k) {
    if ((st = check_rows(k, "k", B, T, D, in_size, out_size, &p.r[1], &kr))) return st;
    st = check_apart(qr.out, "q", kr.out, "the output of k");
    if (!st) st = check_apart(qr.out, "q", kr.x, "k");
    if (!st) st = check_apart(kr.out, "k", qr.x, "q");
    if (st) return st;
  }
  p.B = B;
  p.T = T;
  const hipError_t e = mala::launch_rope(p, D, in_size == 4, out_size == 4, (hipStream_t)stream);
  return e == hipSuccess ? MALA_OK : hip_fail(e, "mala_rope: kernel launch");
}

int mala_paged_rope_write(const mala_rope_rows_t* q, const void* k_new, const void* v_new,
                          int64_t new_token_stride, int64_t new_head_stride, const int32_t* slots,
                          const mala_rope_t* rope, const mala_paged_cache_t* cache, int num_tokens,
                          void* stream) {
  g_err[0] = 0;
  mala::PagedRopeWriteParams p = {};
  int st = check_write(k_new, v_new, new_token_stride, new_head_stride, slots, cache, num_tokens, &p.w);
  if (!st) st = check_turn(rope, 1, num_tokens, cache->D, 0, &p.q.turn);
  if (st || !num_tokens) return st;
  TurnedRows qr;
  if (q) {
    if ((st = check_rows(q, "q", 1, num_tokens, cache->D, 2, 2, &p.q.r[0], &qr))) return st;
    const int64_t n[2] = {cache->Hkv, num_tokens};
    mala::Rows rows = {(uintptr_t)k_new, (int64_t)cache->D * 2, {0, n[0] > 1 ? p.w.head_stride : 0,
                       n[1] > 1 ? p.w.token_stride : 0}, {1, n[0], n[1]}};
    if ((st = check_apart(qr.out, "q", rows, "k_new"))) return st;
    rows.base = (uintptr_t)v_new;
    if ((st = check_apart(qr.out, "q", rows, "v_new"))) return st;
  }
  if ((st = check_scales_apart(p.w.c, cache->D))) return st;
  p.q.B = 1;
  p.q.T = num_tokens;
  // a workgroup per rope_tokens(D) tokens, and per head at most, and those of a block-scaled write; in
  // one dimension
  const double groups = ((double)num_tokens / mala::rope_tokens(cache->D) + 1) *
                            (p.q.r[0].H + 2.0 * cache->Hkv) +
                        (double)mala::block_write_plan(num_tokens, cache->Hkv, true).groups;
  if (groups * 256 > UINT32_MAX) return fail(MALA_ERR_UNSUPPORTED, "a launch of 2^32 threads or more");
  const hipError_t e = mala::launch_paged_rope_write(p, cache->D, (hipStream_t)stream);
  return e == hipSuccess ? MALA_OK : hip_fail(e, "mala_paged_rope_write: kernel launch");
}

int mala_paged_read(const mala_paged_cache_t* cache, const int32_t* block_table,
                    const int32_t* cu_seqlens, void* k, void* v, int num_seqs, int max_pages,
                    int max_seqlen, int total, void* stream) {
  g_err[0] = 0;
  mala::PagedReadParams p;
  int st = check_cache(cache, &p.c);
  if (st) return st;
  if (!block_table || !cu_seqlens || !k || !v)
    return fail(MALA_ERR_INVALID_ARG, "null block_table, cu_seqlens, k or v");
  if (num_seqs <= 0 || max_pages <= 0 || max_seqlen <= 0 || total <= 0)
    return fail(MALA_ERR_INVALID_ARG, "non-positive size (num_seqs, max_pages, max_seqlen, total)");
  if (max_seqlen > (int64_t)max_pages * cache->page_size)
    return fail(MALA_ERR_INVALID_ARG, "max_seqlen (%d) above max_pages x page_size", max_seqlen);
  if ((uintptr_t)k % 16 || (uintptr_t)v % 16) return fail(MALA_ERR_INVALID_ARG, "k or v not 16-byte aligned");
  if ((st = check_slice_range(total, cache->D))) return st;
  p.table = block_table;
  p.cu = cu_seqlens;
  p.k = (char*)k;
  p.v = (char*)v;
  p.S = num_seqs; p.W = max_pages; p.max_len = max_seqlen; p.total = total;
  const hipError_t e = mala::launch_paged_read(p, cache->D, (hipStream_t)stream);
  return e == hipSuccess ? MALA_OK : hip_fail(e, "mala_paged_read: kernel launch");
}

size_t mala_paged_decode_workspace_size(int B, int Hq, int Hkv, int D, int max_len,
                                        int split_tokens) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || (D != 64 && D != 128) || max_len <= 0 ||
      max_len > mala::kPagedMaxLen || split_tokens <= 0 || split_tokens % mala::kDecBk)
    return 0;
  const size_t n = mala::paged_decode_blocks(B, Hq, Hkv, D, max_len, split_tokens);
  if (n <= (size_t)B) return 0;
  return paged_plan_bytes(B) + round_up(n * Hq * (D + mala::kDecStride) * sizeof(float), 256);
}

int mala_paged_decode(const void* q, const mala_paged_cache_t* cache, const int32_t* block_table,
                      const int32_t* cache_lens, void* o, float* lse, int32_t* head_tiles,
                      int64_t* counters, int split_tokens, void* workspace,
                      size_t workspace_bytes, int B, int Hq, int max_pages, int max_len,
                      float scale, float tau, int out_dtype, void* stream) {
  g_err[0] = 0;
  mala::PagedDecParams p;
  int st = check_cache(cache, &p.c);
  if (st) return st;
  if (!q || !block_table || !cache_lens || !o || !lse)
    return fail(MALA_ERR_INVALID_ARG, "null q, block_table, cache_lens, o or lse");
  if (max_pages <= 0) return fail(MALA_ERR_INVALID_ARG, "non-positive max_pages");
  st = check_common(B, Hq, cache->Hkv, 1, max_len, cache->D, 1, scale, tau);
  if (!st) st = check_dtype(out_dtype, "out_dtype");
  if (!st) st = check_split_tokens(split_tokens);
  if (st) return st;
  if (max_len > (int64_t)max_pages * cache->page_size)
    return fail(MALA_ERR_INVALID_ARG, "max_len (%d) above max_pages x page_size", max_len);
  if ((uintptr_t)q % 16 || (uintptr_t)o % 16) return fail(MALA_ERR_INVALID_ARG, "q or o not 16-byte aligned");
  const size_t need =
      mala_paged_decode_workspace_size(B, Hq, cache->Hkv, cache->D, max_len, split_tokens);
  if (need && (!workspace || workspace_bytes < need))
    return fail(MALA_ERR_WORKSPACE, "mala_paged_decode needs %zu workspace bytes, got %zu", need,
                workspace_bytes);
  if (((uintptr_t)workspace) % 16) return fail(MALA_ERR_WORKSPACE, "workspace not 16-byte aligned");
  p.q = (const __bf16*)q;
  p.table = block_table;
  p.lens = cache_lens;
  p.plan = (int2*)workspace;
  p.part = workspace ? (float*)((char*)workspace + paged_plan_bytes(B)) : nullptr;
  p.o = o;
  p.o_bf16 = out_dtype == MALA_OUT_BF16;
  p.lse = lse;
  p.head_tiles = head_tiles;
  p.counters = (unsigned long long*)counters;
  p.B = B; p.Hq = Hq; p.W = max_pages; p.max_len = max_len;
  p.scale2 = scale * mala::kLog2e;
  p.log2tau = log2_tau(tau);
  if (max_len > mala::kPagedMaxLen) return fail(MALA_ERR_UNSUPPORTED, "max_len %d", max_len);
  // (bounds the decode's grid and the join's, of 256 threads per workgroup)
  const double groups =
      (double)(Hq + 8) * mala::paged_decode_blocks(B, Hq, cache->Hkv, cache->D, max_len, split_tokens);
  if (groups * 256 + 65536 > UINT32_MAX || (double)B * max_len / mala::kDecBk > INT32_MAX / 2)
    return fail(MALA_ERR_UNSUPPORTED, "a launch of 2^32 threads or 2^30 tiles, or more");
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (counters &&
      (e = mala::launch_fill_zero(counters, mala::kNumCounters * sizeof(int64_t), s)) != hipSuccess)
    return hip_fail(e, "mala_paged_decode: clearing counters");
  if ((e = mala::launch_paged_decode(p, cache->D, split_tokens, s)) != hipSuccess)
    return hip_fail(e, "mala_paged_decode: kernel launch");
  return MALA_OK;
}

}  // extern "C"
