// Where the loads of the packed microscaled weight begin; host and device, so that the host can hold them against the weight's end.
#pragma once

namespace sqap {

// Bytes from the first of a wavefront's fragments to stage `stage` of fragment `fragment`, `bytes` of each a stage.  A kernel asks for stages ahead
// of the one that it multiplies, up to its depth past the last: those are the last one once more, whose loads stay inside (a buffer's range is
// checked against a lane's offset; this one is the wavefront's).
__host__ __device__ static inline unsigned weight_stage(int fragment, int stage, int stages, unsigned bytes)
{
    return (unsigned)(fragment * stages + (stage < stages ? stage : stages - 1)) * bytes;
}

}  // namespace sqap
