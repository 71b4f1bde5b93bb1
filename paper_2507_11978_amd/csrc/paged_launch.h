// Launches of the paged attention kernels for one built head size (host side).
#pragma once
#include "paged_few.h"
#include "paged_many.h"

namespace nt {

template <typename Kernel>
static nt_status launch_paged_inst(Kernel kern, DeviceOnce &configured, const char *name, size_t lds, const PagedArgs &a, int64_t programs, hipStream_t s)
{
    if (lds > 65536 && !configured.done()) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return fail(NT_ERR_DEVICE, std::string("hipFuncSetAttribute: ") + hipGetErrorString(e));
        configured.set();
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)programs), dim3(256), lds, s, a);
    return check_launch(name);
}

template <int SIZE, bool BF16, int KIND, int MB>
static nt_status launch_paged_few(const PagedArgs &a, int64_t programs, hipStream_t s)
{
    static DeviceOnce c[3];
    const char *name = "paged_few_kernel";
    if (a.uniform && a.D == SIZE) return launch_paged_inst(paged_few_kernel<BF16, KIND, SIZE, MB, true, true>, c[0], name, few_lds(SIZE, MB), a, programs, s);
    if (a.uniform) return launch_paged_inst(paged_few_kernel<BF16, KIND, SIZE, MB, true, false>, c[1], name, few_lds(SIZE, MB), a, programs, s);
    return launch_paged_inst(paged_few_kernel<BF16, KIND, SIZE, MB, false, false>, c[2], name, few_lds(SIZE, MB), a, programs, s);
}

template <int SIZE, bool BF16, int KIND>
static nt_status launch_paged_kind(const PagedArgs &a, int rows, int64_t programs, hipStream_t s)
{
    static_assert(kFewWaves == 4 && kManyWaves == 4, "256 threads");
    static DeviceOnce many[3];
    if (rows == 16) return launch_paged_few<SIZE, BF16, KIND, 1>(a, programs, s);
    if constexpr (SIZE < 256)                                              // (two sets of 16 rows of 256 elements do not fit the registers)
        if (rows == 32) return launch_paged_few<SIZE, BF16, KIND, 2>(a, programs, s);
    const bool together = a.near && a.aligned && a.page.d % many_together(KIND, SIZE) == 0 && a.D % many_piece(KIND) == 0;
    const char *name = "paged_many_kernel";
    if (together && a.D == SIZE) return launch_paged_inst(paged_many_kernel<BF16, KIND, SIZE, true, true>, many[0], name, many_lds(SIZE), a, programs, s);
    if (together) return launch_paged_inst(paged_many_kernel<BF16, KIND, SIZE, true, false>, many[1], name, many_lds(SIZE), a, programs, s);
    return launch_paged_inst(paged_many_kernel<BF16, KIND, SIZE, false, false>, many[2], name, many_lds(SIZE), a, programs, s);
}

// rows: to a program, 16, 32 (paged_few_kernel) or kManyRows
template <int SIZE>
static nt_status launch_paged_size(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (kind == CACHE_E4M3) return bf16 ? launch_paged_kind<SIZE, true, CACHE_E4M3>(a, rows, programs, s) : launch_paged_kind<SIZE, false, CACHE_E4M3>(a, rows, programs, s);
    if (kind == CACHE_I8) return bf16 ? launch_paged_kind<SIZE, true, CACHE_I8>(a, rows, programs, s) : launch_paged_kind<SIZE, false, CACHE_I8>(a, rows, programs, s);
    return bf16 ? launch_paged_kind<SIZE, true, CACHE_SAME>(a, rows, programs, s) : launch_paged_kind<SIZE, false, CACHE_SAME>(a, rows, programs, s);
}

}  // namespace nt
