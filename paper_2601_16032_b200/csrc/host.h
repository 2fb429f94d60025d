// What the library's host files share: the error text of the calling thread, what is known about the current device.
#pragma once
#include <cuda_runtime.h>

#include "../../include/sawtooth_attn.h"

namespace sawtooth {

constexpr int kMaxDevices = 64;

// Codes of the device status word at and above this one say that a kernel met an index out of range; below it, that a
// wait ran out (WaitSite).
constexpr int kFirstIndexCode = 64;
enum IndexSite { kIndexLength = 64, kIndexPage = 65, kIndexSlot = 66 };

// What the library knows about a device, looked up once (under a mutex) on the first call that has it current: its
// size, the device addresses of the library's own __device__ variables there, and which kernel variants have had their
// dynamic shared memory limit raised.  Readers take a copy under the same mutex.
struct DeviceState {
    bool ready = false;
    int sm_count = 0, smem_optin = 0;
    int* status = nullptr;
    unsigned long long* cycles = nullptr;
    int* noalloc_scratch = nullptr;
    unsigned smem_raised = 0;   // bit v: variant v of the forward kernel may use smem_optin bytes
    unsigned paged_raised = 0;  // the same for the kernels of paged.cu, each with a limit of its own
};

// Notes the text of an error for attn_last_error and returns `status`.
int fail(int status, const char* fmt, ...);
// The current device's state, filled on first use.  *dev_out, if given, gets the device index.
int current_device(DeviceState* out, int* dev_out);
// Allows `kernel` that many bytes of dynamic shared memory, once per device and bit of paged_raised.
int raise_smem(int dev, const DeviceState& ds, const void* kernel, int bit, int bytes);
// Reads and clears the current device's status word after a device synchronisation.
int read_status(int* code);

}  // namespace sawtooth
