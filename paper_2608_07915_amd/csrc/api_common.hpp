// Checks and error texts shared by the C entry points that run on the GPU.
#pragma once
#include <hip/hip_runtime.h>

#include "host_common.hpp"

namespace spectra {

inline spectra_status hip_fail(hipError_t e, const char* what) {
  return fail(SPECTRA_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline spectra_status check_codec(const spectra_codec* c, const char* name, bool layer_ok = false) {
  if (!c) return fail(SPECTRA_EINVAL, "%s: null codec", name);
  spectra_status st = check_params_gpu(c->p);
  if (st != SPECTRA_OK) return st;
  if (!layer_ok && layer_geometry(c->p))
    return fail(SPECTRA_EUNSUPPORTED, "%s: the per-layer geometry (head_dim %d, group_size 64) supports fit, encode and decode only",
                name, c->p.head_dim);
  if (c->record_words != record_words(c->p))
    return fail(SPECTRA_EINVAL, "%s: record_words %d does not match the parameters (%d); call spectra_codec_init",
                name, c->record_words, record_words(c->p));
  if (c->n_streams <= 0 || c->n_streams > 65535)
    return fail(SPECTRA_EINVAL, "%s: n_streams=%lld out of range [1, 65535]", name, (long long)c->n_streams);
  if (!c->basis || !c->mean || !c->var || !c->bits) return fail(SPECTRA_EINVAL, "%s: null codec array", name);
  if (c->lscale && !layer_geometry(c->p))
    return fail(SPECTRA_EUNSUPPORTED, "%s: the square-root latent split (lscale) runs in the per-layer geometry only", name);
  if (c->lscale && !aligned(c->lscale, 4)) return fail(SPECTRA_EINVAL, "%s: lscale must be 4-byte aligned", name);
  if (!aligned(c->basis, 16) || !aligned(c->mean, 4) || !aligned(c->var, 4) || !aligned(c->bits, 4))
    return fail(SPECTRA_EINVAL, "%s: basis must be 16-byte aligned, the other codec arrays 4-byte aligned", name);
  return SPECTRA_OK;
}

inline size_t round256(size_t b) { return (b + 255) / 256 * 256; }

}  // namespace spectra
