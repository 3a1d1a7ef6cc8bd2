// The launchers of the operators in mergecomp_step.h as their host code sees them, without a device: each notes that it was called and with how many
// rows or pieces.  Linked with step_api.hip and no_device.hip (the runtime).
#include <cstring>
#include <string>

#include "../../paper_2103_15195_amd/csrc/step_internal.h"

static std::string g_log;

extern "C" {
const char *nds_log(void) { return g_log.c_str(); }
void nds_forget(void) { g_log.clear(); }
hipError_t hipLaunchKernel(const void *, dim3, dim3, void **, size_t, hipStream_t) { return hipErrorNotSupported; }
}

namespace mc {
static void note(const char *what, uint64_t n) { g_log += std::string(what) + ":" + std::to_string(n) + " "; }
void launch_grad_norm(const LaunchCtx &, int, const StepView &v, double *, uint32_t *, float, float, float *) { note("norm", v.npieces); }
void launch_grad_clip(const LaunchCtx &, int, const StepView &, uint32_t to_list, const float *) { note("clip", to_list); }
void launch_adamw(const LaunchCtx &, int, int model_dtype, const StepView &v, const AdamwArgs &) { note(model_dtype < 0 ? "adamw" : "adamw+copy", v.npieces); }
void launch_token_logp(const LaunchCtx &, int, const LossArgs &a) { note("logp", a.rows); }
void launch_policy_loss(const LaunchCtx &, int, const LossArgs &a) { note("policy", a.rows); }
}  // namespace mc
