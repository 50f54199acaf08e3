// Library-wide entry points: device error word, status names, version.
#include <cuda_runtime.h>

#include "common.cuh"

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_attn_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_score_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_loss_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_kv_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_rope_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_prompt_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_trunc_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_kv8_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_attn8_error();
extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_draft_error();

extern "C" int ipd_get_device_error(uint32_t *code) {
  if (!code) return IPD_ERR_INVALID_ARG;
  if (cudaDeviceSynchronize() != cudaSuccess) return IPD_ERR_CUDA;
  // every word is taken (and cleared) before one is returned; the first wins
  const unsigned int words[] = {ipd_internal_take_attn_error(), ipd_internal_take_score_error(),
                                ipd_internal_take_loss_error(), ipd_internal_take_kv_error(),
                                ipd_internal_take_rope_error(), ipd_internal_take_prompt_error(),
                                ipd_internal_take_trunc_error(), ipd_internal_take_kv8_error(),
                                ipd_internal_take_attn8_error(), ipd_internal_take_draft_error()};
  unsigned int first = 0;
  for (const unsigned int w : words) {
    if (w == 0xffffffffu) return IPD_ERR_CUDA;
    if (first == 0) first = w;
  }
  *code = first;
  return IPD_OK;
}

extern "C" const char *ipd_status_string(int status) {
  switch (status) {
    case IPD_OK: return "IPD_OK";
    case IPD_ERR_INVALID_ARG: return "IPD_ERR_INVALID_ARG";
    case IPD_ERR_UNSUPPORTED: return "IPD_ERR_UNSUPPORTED";
    case IPD_ERR_WORKSPACE: return "IPD_ERR_WORKSPACE";
    case IPD_ERR_CUDA: return "IPD_ERR_CUDA";
    case IPD_ERR_TIMEOUT: return "IPD_ERR_TIMEOUT";
    case IPD_ERR_DEVICE: return "IPD_ERR_DEVICE";
    case IPD_ERR_CAPACITY: return "IPD_ERR_CAPACITY";
    default: return "IPD_ERR_UNKNOWN";
  }
}

extern "C" int ipd_version(void) { return 100; }

extern "C" int ipd_device_readable(const void *ptr, int *readable) {
  if (!readable) return IPD_ERR_INVALID_ARG;
  *readable = 0;
  if (!ptr) return IPD_OK;
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, ptr) != cudaSuccess) {
    (void)cudaGetLastError();  // an unregistered host pointer is not an error state
    return IPD_OK;
  }
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return IPD_ERR_CUDA;
  if (a.type == cudaMemoryTypeDevice) *readable = a.device == dev;
  else if (a.type == cudaMemoryTypeManaged) *readable = 1;
  else if (a.type == cudaMemoryTypeHost) *readable = a.devicePointer == ptr;
  return IPD_OK;
}
