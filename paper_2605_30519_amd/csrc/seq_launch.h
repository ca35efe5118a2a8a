// seq_launch.h -- host-side launchers of the sequence cache's kernels (internal to the library).
#pragma once

#include <hip/hip_runtime.h>

#include "seq.h"

namespace omnimem {

hipError_t launch_decode(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, void* workspace,
                         hipStream_t stream);
hipError_t launch_append_kv(const SeqGeom& g, const AppendLaunch& a, hipStream_t stream);
hipError_t launch_copy_pages(const CopyLaunch& a, hipStream_t stream);
hipError_t launch_decode_quant(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, void* workspace,
                               hipStream_t stream);
hipError_t launch_append_kv_quant(const SeqGeom& g, const AppendQuantLaunch& a, hipStream_t stream);
hipError_t launch_read_kv_quant(const SeqGeom& g, const ReadQuantLaunch& a, hipStream_t stream);
hipError_t launch_seq_update(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, void* workspace,
                             hipStream_t stream);
hipError_t launch_seq_compact(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, void* workspace,
                              hipStream_t stream);

}  // namespace omnimem
