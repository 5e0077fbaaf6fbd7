// Entry points of token sampling: argument checks and the choice between the two kernel families.

#include "sample.cuh"

using namespace a3po;

extern "C" {

size_t a3po_sample_workspace_bytes(int64_t N, int V) {
  if (N < 0 || V <= 0 || N > INT_MAX) return 0;
  return sample_stream_bytes(N, V) + 256;
}

int a3po_sample(const void* logits, int64_t row_stride, const uint8_t* row_mask, int64_t N, int V, a3po_dtype dt,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                int32_t* token, float* logp, float* kept_logp, int32_t* n_kept, void* ws, size_t ws_bytes,
                void* stream) {
  if (N < 0 || V <= 0 || (N > 1 && row_stride < V)) return A3PO_ERR_INVALID_ARG;
  if (dt != A3PO_F32 && dt != A3PO_BF16) return A3PO_ERR_UNSUPPORTED;
  if (N > 0 && (!logits || !u || !token)) return A3PO_ERR_INVALID_ARG;
  if (N > INT_MAX || V > INT_MAX - 4096) return A3PO_ERR_UNSUPPORTED;
  if (!aligned_to(logits, dt == A3PO_F32 ? 4 : 2)) return A3PO_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(temperature), static_cast<const void*>(top_k), static_cast<const void*>(top_p),
                        static_cast<const void*>(min_p), static_cast<const void*>(u), static_cast<const void*>(token),
                        static_cast<const void*>(logp), static_cast<const void*>(kept_logp), static_cast<const void*>(n_kept)})
    if (!aligned_to(p, 4)) return A3PO_ERR_UNSUPPORTED;
  const bool filters = top_k || top_p || min_p;
  if (filters && V > sample_filter_max_v(dt)) return A3PO_ERR_UNSUPPORTED;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < a3po_sample_workspace_bytes(N, V)) return A3PO_ERR_WORKSPACE;
  if (sm_count() <= 0) return A3PO_ERR_NO_DEVICE;
  if (N == 0) return A3PO_OK;
  const SampleArgs a{logits, row_stride, row_mask, static_cast<int>(N), V, temperature, top_k, top_p, min_p, u,
                     token, logp, kept_logp, n_kept};
  return filters || sample_in_one(N, V) ? sample_filter(&a, dt, as_stream(stream)) : sample_stream(&a, dt, ws, as_stream(stream));
}

}  // extern "C"
