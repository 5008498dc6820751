// C entry points of the 8-bit paged KV cache: argument checks and launches.
#include <mutex>

#include "paged.cuh"

namespace {

using namespace dvi;

// Multiprocessors of the current device, looked up once per device.
int current_sms() {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> sms[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  int n = dev < kMaxDevices ? sms[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < kMaxDevices) sms[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Query vectors (rows x query heads of a KV head) up to which a bf16 sequence's rows are
// few.  Which kernel is faster depends on the lengths too, and those are on the device:
// the border is where a wrong choice costs least.  us by the few-row kernel / the prompt
// kernel, int8 and 8 KV heads of 128: below it 24 vectors over 200 positions 12.1 / 11.4
// (8 sequences), 28 over 16000 26.1 / 32.2 (1), 24 over 4000 71.5 / 160 (32), 32 over 500
// 16.3 / 28.2 (32, hd 64); above it, one sequence, 40 over 20 10.8 / 7.9, 64 over 500
// 17.3 / 15.6, 40 over 4000 19.0 / 20.2, 64 over 16000 31.0 / 36.1.
constexpr int kFewVectors = 32;

// Held while an attend is enqueued: the second launch of a mixed batch runs beside the one before
// it on its stream, which has to be its own first one and not another host thread's attend, as
// that one shares its counters.  One lock for each of 64 kinds of stream handles.
std::mutex& enqueue_lock(dvi_stream stream) {
  static std::mutex locks[64];
  return locks[(reinterpret_cast<uintptr_t>(stream) * 0x9e3779b97f4a7c15ull) >> 58];
}

bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool ld_ok(int64_t ld, int64_t least, int esz) { return ld >= least && (ld * esz) % 16 == 0; }

// DVI_OK, or what is wrong with the cache and the batch.
dvi_status check(const dvi_paged_cache* c, const dvi_paged_batch* b, int dtype, PagedArgs* out) {
  if (!c || !b || (dtype != DVI_F32 && dtype != DVI_BF16)) return DVI_ERR_INVALID_ARG;
  const int P = c->page_tokens;
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || (P != 16 && P != 32 && P != 64 && P != 128) ||
      (c->head_dim != 64 && c->head_dim != 128) || (c->format != DVI_KV_INT8 && c->format != DVI_KV_E4M3))
    return DVI_ERR_INVALID_ARG;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !on16(c->k) || !on16(c->v) || !on16(c->k_scale) ||
      !on16(c->v_scale))
    return DVI_ERR_INVALID_ARG;
  if (b->n_seqs < 1 || b->max_pages < 1 || b->n_rows < 0 || b->max_rows < 0 || !b->table || !b->lens)
    return DVI_ERR_INVALID_ARG;
  if (!b->row_start && b->n_rows % b->n_seqs) return DVI_ERR_INVALID_ARG;
  if (!b->row_start && b->max_rows < b->n_rows / b->n_seqs) return DVI_ERR_INVALID_ARG;
  // positions and row counts are 32-bit numbers on the device
  if (b->n_seqs > kPagedMaxSeqs || static_cast<int64_t>(b->max_pages) * P > (1ll << 30) || b->n_rows > (1 << 30))
    return DVI_ERR_CAPACITY;
  PagedArgs a{};
  a.k = static_cast<uint8_t*>(c->k);
  a.v = static_cast<uint8_t*>(c->v);
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.table = b->table;
  a.lens = b->lens;
  a.row_start = b->row_start;
  a.status = b->status;
  a.n_pages = c->n_pages;
  a.H = c->n_kv_heads;
  a.P = P;
  a.log_p = P == 16 ? 4 : P == 32 ? 5 : P == 64 ? 6 : 7;
  a.D = c->head_dim;
  a.n_seqs = b->n_seqs;
  a.max_pages = b->max_pages;
  a.n_rows = b->n_rows;
  // (a bound, and what the launches are chosen by: without row starts the count itself is known)
  a.max_rows = !b->row_start ? b->n_rows / b->n_seqs : b->max_rows < b->n_rows ? b->max_rows : b->n_rows;
  *out = a;
  return DVI_OK;
}

// The launchers refuse grids and unit counts past 31 bits.
dvi_status launched(cudaError_t e) {
  return e == cudaSuccess ? DVI_OK : e == cudaErrorInvalidConfiguration ? DVI_ERR_CAPACITY : DVI_ERR_CUDA;
}

}  // namespace

extern "C" dvi_status dvi_paged_append(const dvi_paged_cache* cache, const dvi_paged_batch* batch, int dtype,
                                       const void* d_k, int64_t ld_k, const void* d_v, int64_t ld_v,
                                       const float* d_rotary, int rot_dim, int n_pos, const void* d_q, int64_t ld_q,
                                       void* d_q_out, int64_t ld_q_out, int n_heads, dvi_stream stream) {
  PagedAppendArgs a{};
  const dvi_status rc = check(cache, batch, dtype, &a.c);
  if (rc != DVI_OK) return rc;
  if (a.c.n_rows == 0) return DVI_OK;
  const int esz = dtype == DVI_F32 ? 4 : 2;
  const int64_t kv = static_cast<int64_t>(a.c.H) * a.c.D;
  if (!d_k || !d_v || !on16(d_k) || !on16(d_v) || !ld_ok(ld_k, kv, esz) || !ld_ok(ld_v, kv, esz))
    return DVI_ERR_INVALID_ARG;
  if (d_rotary && (rot_dim < 16 || rot_dim > a.c.D || rot_dim % 16 || n_pos < 1 || !on16(d_rotary)))
    return DVI_ERR_INVALID_ARG;
  if (d_q) {
    const int64_t least = static_cast<int64_t>(n_heads) * a.c.D;
    if (n_heads < 1 || n_heads > (1 << 16) || !d_q_out || !on16(d_q) || !on16(d_q_out) || !ld_ok(ld_q, least, esz) ||
        !ld_ok(ld_q_out, least, esz))
      return DVI_ERR_INVALID_ARG;
  }
  a.kin = d_k;
  a.vin = d_v;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.rotary = reinterpret_cast<const float2*>(d_rotary);
  a.rot = d_rotary ? rot_dim : 0;
  a.n_pos = n_pos;
  a.q = d_q;
  a.q_out = d_q_out;
  a.ld_q = ld_q;
  a.ld_qo = ld_q_out;
  a.n_heads = n_heads;
  a.dtype = dtype;
  cudaGetLastError();   // an error left pending by the caller is not this call's
  return launched(launch_paged_append(a, cache->format == DVI_KV_E4M3, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" dvi_status dvi_paged_attend(const dvi_paged_cache* cache, const dvi_paged_batch* batch,
                                       const dvi_paged_options* options, int dtype, const void* d_q, int64_t ld_q,
                                       void* d_o, int64_t ld_o, void* workspace, size_t workspace_bytes,
                                       dvi_stream stream) {
  PagedAttendArgs a{};
  const dvi_status rc = check(cache, batch, dtype, &a.c);
  if (rc != DVI_OK) return rc;
  const int esz = dtype == DVI_F32 ? 4 : 2;
  if (!options || options->n_heads < 1 || options->n_heads > (1 << 16) || options->n_heads % a.c.H ||
      !(options->scale > 0.f) || !(options->scale < 1e30f) || !(options->softcap >= 0.f) ||
      !(options->softcap < 1e30f) || options->window < 0)
    return DVI_ERR_INVALID_ARG;
  if (options->softcap > 0.f && !(options->scale / options->softcap < 1e30f)) return DVI_ERR_INVALID_ARG;
  if (a.c.n_rows == 0) return DVI_OK;
  const int64_t least = static_cast<int64_t>(options->n_heads) * a.c.D;
  if (!d_q || !d_o || !on16(d_q) || !on16(d_o) || !ld_ok(ld_q, least, esz) || !ld_ok(ld_o, least, esz))
    return DVI_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return DVI_ERR_INVALID_ARG;
  if (static_cast<int64_t>(a.c.n_rows) * (options->n_heads / a.c.H) > 0x7fffffffll) return DVI_ERR_CAPACITY;
  const int sms = current_sms();
  if (sms <= 0) return DVI_ERR_CUDA;
  if (workspace_bytes < dvi_paged_workspace_bytes(a.c.D)) return DVI_ERR_CAPACITY;
  a.q = d_q;
  a.o = d_o;
  a.ld_q = ld_q;
  a.ld_o = ld_o;
  a.slopes = options->slopes;
  a.n_heads = options->n_heads;
  a.G = options->n_heads / a.c.H;
  a.inv_g = a.G == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + a.G - 1) / a.G);
  a.dtype = dtype;
  a.scale = options->scale;
  if (dtype == DVI_BF16 && options->softcap > kPagedPlainCap) {
    const float top = options->softcap * 1.4426950408889634f;
    a.cap = {1.f / top, 2.f / options->softcap, top, 0.25f * top};
  } else {
    a.softcap = options->softcap;
  }
  a.window = options->window < (1 << 30) ? options->window : 0;   // no position is further back
  a.counters = static_cast<int*>(workspace);
  a.pf_counters = a.counters + static_cast<size_t>(sms) * kPagedTeams;
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + paged_counter_bytes(sms));
  a.pf_part = a.part + paged_part_floats(a.c.D, sms);
  std::lock_guard<std::mutex> enqueue(enqueue_lock(stream));
  cudaGetLastError();
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool e4m3 = cache->format == DVI_KV_E4M3;
  // Row starts lie on the device and max_rows only bounds them, so any of their sequences may
  // hold few rows.  Of several, each launch skips the other's; a single sequence is the
  // prompt kernel's whatever it holds (both launches / that one, us: 1000 rows behind 20 to
  // 16000 positions 4 to 13 more of 28 to 333; 1 row in a buffer of 64, 8 KV heads, 14.6 / 11.8
  // behind 540 and 20.5 / 24.9 behind 16000, 32 KV heads 46.9 / 85.2).
  const int64_t most = static_cast<int64_t>(a.c.max_rows) * a.G;
  const bool prompts = dtype == DVI_BF16 && a.G <= 128 && most > kFewVectors;
  const bool few = !prompts || (a.c.row_start && a.c.n_seqs > 1);
  if (prompts) {
    a.min_vectors = few ? kFewVectors + 1 : 1;
    a.max_vectors = 0x7fffffff;
    const dvi_status r = launched(launch_paged_pf(a, e4m3, sms, st));
    if (r != DVI_OK) return r;
  }
  if (few) {
    a.min_vectors = 1;
    a.max_vectors = prompts ? kFewVectors : 0x7fffffff;
    a.beside = prompts;
    return launched(e4m3 ? launch_paged_attend<true>(a, sms, st) : launch_paged_attend<false>(a, sms, st));
  }
  return DVI_OK;
}

extern "C" size_t dvi_paged_workspace_bytes(int head_dim) {
  const int sms = current_sms();
  if ((head_dim != 64 && head_dim != 128) || sms <= 0) return 0;
  return paged_counter_bytes(sms) +
         (paged_part_floats(head_dim, sms) + paged_pf_part_floats(head_dim, sms)) * sizeof(float);
}

extern "C" size_t dvi_paged_counter_bytes(void) {
  const int sms = current_sms();
  return sms > 0 ? paged_counter_bytes(sms) : 0;
}

extern "C" uint64_t dvi_paged_capture(dvi_stream stream) {
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (cudaStreamGetCaptureInfo(reinterpret_cast<cudaStream_t>(stream), &status, &id) != cudaSuccess) {
    cudaGetLastError();   // (the legacy stream while another is captured: a launch there says so)
    return 0;
  }
  return status == cudaStreamCaptureStatusNone ? 0 : id;
}

extern "C" dvi_status dvi_paged_read(const dvi_paged_cache* cache, const dvi_paged_batch* batch, int dtype,
                                     void* d_k_out, void* d_v_out, dvi_stream stream) {
  PagedReadArgs a{};
  const dvi_status rc = check(cache, batch, dtype, &a.c);
  if (rc != DVI_OK) return rc;
  if (a.c.n_rows == 0) return DVI_OK;
  if (!d_k_out || !d_v_out || !on16(d_k_out) || !on16(d_v_out)) return DVI_ERR_INVALID_ARG;
  a.k_out = d_k_out;
  a.v_out = d_v_out;
  a.dtype = dtype;
  cudaGetLastError();
  return launched(launch_paged_read(a, cache->format == DVI_KV_E4M3, reinterpret_cast<cudaStream_t>(stream)));
}
