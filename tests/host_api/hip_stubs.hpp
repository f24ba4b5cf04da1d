// The library's C-ABI layer as host code: the HIP runtime's few calls as host memory, launches that are counted and can be made to fail.
#pragma once

#include "../../paper_2603_17051_amd/csrc/astro_api.hip"

#include <cstdlib>

inline int launches = 0;
inline bool launches_fail = false;
inline hipError_t launched() {
  ++launches;
  return launches_fail ? hipErrorInvalidConfiguration : hipSuccess;
}

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipMemcpy(void* to, const void* from, size_t n, hipMemcpyKind) { return std::memcpy(to, from, n), hipSuccess; }
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { return launched(); }
hipError_t hipGetLastError() { return hipSuccess; }
}

namespace astro {
ProfileScope::ProfileScope(const char*, hipStream_t, bool) {}
ProfileScope::~ProfileScope() {}
size_t f32_fwd_workspace_floats(const DevGeom&, int) { return 0; }
size_t f32_bwd_workspace_floats(const DevGeom&, int) { return 0; }
size_t bf16_fwd_split_bytes(const DevGeom&, int) { return 0; }
size_t bf16_bwd_workspace_bytes(const DevGeom&, int) { return 256; }
size_t select_fwd_split_bytes(const DevGeom&, int) { return 256; }
size_t select_bwd_bytes(const DevGeom&, int) { return 256; }
bool bf16_fwd_rotates(const DevGeom&, const AttnOperands&) { return false; }
bool bf16_bwd_joins(const DevGeom&, const AttnOperands&) { return false; }
hipError_t launch_rope_scatter(const DevGeom&, int, const void*, const void*, ScatterDst, bool, int, const StreamInts&, const StreamInts&, float2*, float,
                               hipStream_t) {
  return launched();
}
hipError_t launch_rope_unscatter_f32(const DevGeom&, const float*, float*, int, const StreamInts&, hipStream_t) { return launched(); }
hipError_t launch_rope_sink_rerotate(const DevGeom&, int, const void*, void*, const StreamInts&, const StreamInts&, hipStream_t) { return launched(); }
hipError_t launch_attn_fwd_f32(const DevGeom&, const AttnOperands&, float*, float*, float*, hipStream_t) { return launched(); }
hipError_t launch_attn_bwd_f32(const DevGeom&, const AttnOperands&, const float*, const float*, const float*, float*, float*, float*, float*, hipStream_t) {
  return launched();
}
hipError_t launch_attn_fwd_bf16(const DevGeom&, const AttnOperands&, void*, float*, void*, hipStream_t) { return launched(); }
hipError_t launch_attn_bwd_bf16(const DevGeom&, const AttnOperands&, const void*, const float*, const void*, float*, float*, float*, void*, bool, hipStream_t) {
  return launched();
}
hipError_t launch_attn_bwd_hist_bf16(const DevGeom&, const AttnOperands&, const float*, const void*, float*, float*, float*, float*, const StreamInts&,
                                     const StreamInts&, const StreamInts&, const void*, hipStream_t) {
  return launched();
}
hipError_t launch_kvcache_fork(const ForkArrays&, const ForkPlan&, hipStream_t) { return launched(); }
hipError_t launch_block_means_f32(const DevGeom&, const void*, float*, int, int, const StreamInts&, hipStream_t) { return launched(); }
hipError_t launch_append_means_bf16(const DevGeom&, const void*, const void*, void*, void*, float*, int, int, const StreamInts&, const StreamInts&,
                                    hipStream_t) {
  return launched();
}
hipError_t launch_select_blocks(const DevGeom&, int, const void*, const float*, int, int, int, int, int, const StreamInts&, int32_t*, hipStream_t) {
  return launched();
}
hipError_t launch_select_stage(const DevGeom&, const void*, const void*, const SelectStaged&, int, const StreamInts&, float, hipStream_t) { return launched(); }
hipError_t launch_select_fwd_bf16(const DevGeom&, const AttnOperands&, const SelectStaged&, const SelectLists&, void*, float*, float*, hipStream_t) {
  return launched();
}
hipError_t launch_select_bwd_bf16(const DevGeom&, const AttnOperands&, const SelectStaged&, const SelectLists&, const void*, const float*, const void*, float*,
                                  float*, float*, float*, hipStream_t) {
  return launched();
}
hipError_t launch_select_fwd_f32(const DevGeom&, const AttnOperands&, const SelectLists&, float*, float*, hipStream_t) { return launched(); }
hipError_t launch_select_bwd_f32(const DevGeom&, const AttnOperands&, const SelectLists&, const float*, const float*, const float*, float*, float*, float*,
                                 float*, hipStream_t) {
  return launched();
}
}  // namespace astro
