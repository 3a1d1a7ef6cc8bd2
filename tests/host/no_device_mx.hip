// The launchers of the operators in mergecomp_mx.h as their host code sees them, without a device: each notes that it was called and with what.  Linked with
// mx_api.hip and no_device.hip (the runtime).
#include <cstring>
#include <string>

#include "../../paper_2103_15195_amd/csrc/mx_internal.h"

static std::string g_log;

extern "C" {
const char *ndm_log(void) { return g_log.c_str(); }
void ndm_forget(void) { g_log.clear(); }
hipError_t hipLaunchKernel(const void *, dim3, dim3, void **, size_t, hipStream_t) { return hipErrorNotSupported; }
}

namespace mc {
static void note(const std::string &what) { g_log += what + " "; }
static std::string n(uint64_t x) { return std::to_string(x); }
void launch_adamw8(const LaunchCtx &, int, int model_dtype, const Step8View &v, const AdamwArgs &) { note((model_dtype < 0 ? "adamw8:" : "adamw8+copy:") + n(v.npieces)); }
void launch_mx_quantize(const LaunchCtx &, int, const MxSource &s)
{
    note("quantize:" + n(s.rows) + "x" + n(s.cols) + (s.by_rows.codes ? "r" + n(s.by_rows.steps) : "") + (s.by_cols.codes ? "c" + n(s.by_cols.steps) : "") + (s.values ? "v" : ""));
}
void launch_mx_matmul(const LaunchCtx &, int, const MxProduct &p)
{
    note("matmul:" + n(p.a.rows) + "x" + n(p.b.rows) + "x" + n(p.a.steps) + (p.bias ? "b" : "") + (p.accumulate ? "+" : ""));
}
}  // namespace mc
