// The handle behind the C ABI of include/fa.h and the host helpers that the library's translation units share:
// device guard, tensor-map cache, shared-memory limits.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <vector>

#include "../../include/fa.h"

namespace fa_host {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                   const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct MapEntry {
    const void* ptr;
    int d, S, H, B, box_rows, box_heads, elem_bytes, swizzle_bytes, promotion;
    long long sb, sh, ss;      // batch / head / row strides in elements
    uint64_t stamp;
    CUtensorMap map;
};

constexpr int kMapCacheSize = 16;

}  // namespace fa_host

struct fa_handle {
    int device = 0;
    int num_sms = 1;
    uint32_t flags = 0;
    uint32_t* status_host = nullptr;   // pinned + mapped: [0] status, [1] wait site, [2] kind of bad contents (0: none)
    uint32_t* status_dev = nullptr;
    uint32_t kv_splits_cfg = 0;              // 0 auto, 1 never, n force
    void* scratch = nullptr;                 // split-KV partials
    unsigned int* sched_counter = nullptr;   // work-item ticket counter of the persistent kernel
    unsigned int* arrivals = nullptr;        // paged kernel: finished pieces of a shared row block, one counter per SM (zero between launches)
    size_t scratch_bytes = 0;
    size_t tree_scratch_bytes = 0;           // of the same buffer, what attention of drafted tokens may use
    int last_splits = 1;
    unsigned long long wait_limit_ns = 2000ull * 1000000ull;
    fa_host::EncodeTiledFn encode = nullptr;
    std::vector<fa_host::MapEntry> maps;
    uint64_t stamp = 0;
    uint64_t launches = 0;
    const char* last_kernel = "";
    void* stage[5] = {nullptr, nullptr, nullptr, nullptr, nullptr};   // Q K V O lse
    size_t stage_cap[5] = {0, 0, 0, 0, 0};
    // fa_forward_host on large problems: copy streams and events of the chunked pipeline (created on first use)
    cudaStream_t copy_in = nullptr, copy_out = nullptr;
    cudaEvent_t ev_start = nullptr, ev_out_done = nullptr;
    std::vector<cudaEvent_t> ev_in, ev_done;
    std::vector<const void*> attr_done;     // kernels whose shared-memory limit has been raised
#ifdef FA_TRACE
    long long* trace = nullptr;
#endif
};

namespace fa_host {

class DeviceGuard {
  public:
    explicit DeviceGuard(int want) {
        if (cudaGetDevice(&prev_) != cudaSuccess) prev_ = -1;
        if (prev_ != want) { ok_ = (cudaSetDevice(want) == cudaSuccess); changed_ = ok_; }
    }
    ~DeviceGuard() { if (changed_ && prev_ >= 0) cudaSetDevice(prev_); }
    bool ok() const { return ok_; }
  private:
    int prev_ = -1;
    bool ok_ = true;
    bool changed_ = false;
};

// Tensor of bf16 (elem_bytes 2) or e4m3 (elem_bytes 1) with element (b, h, s, c) at
// ptr + b*sb + h*sh + s*ss + c, seen as a 4-D TMA tensor (d, S, H, B); box = 128 bytes of columns
// x box_rows rows, 128-byte swizzle, rows past S read as zero.
inline fa_status get_map(fa_handle* h, const void* ptr, int d, int S, int H, int B, long long sb, long long sh,
                  long long ss, int box_rows, const CUtensorMap** out, int elem_bytes = 2, int box_heads = 1,
                  int swizzle_bytes = 128, int promotion = CU_TENSOR_MAP_L2_PROMOTION_L2_256B) {
    for (auto& e : h->maps) {
        if (e.ptr == ptr && e.d == d && e.S == S && e.H == H && e.B == B && e.box_rows == box_rows &&
            e.sb == sb && e.sh == sh && e.ss == ss && e.elem_bytes == elem_bytes && e.box_heads == box_heads && e.swizzle_bytes == swizzle_bytes && e.promotion == promotion) {
            e.stamp = ++h->stamp;
            *out = &e.map;
            return FA_OK;
        }
    }
    MapEntry ne;
    memset(&ne, 0, sizeof ne);
    ne.ptr = ptr; ne.d = d; ne.S = S; ne.H = H; ne.B = B; ne.box_rows = box_rows;
    ne.sb = sb; ne.sh = sh; ne.ss = ss; ne.elem_bytes = elem_bytes; ne.box_heads = box_heads; ne.swizzle_bytes = swizzle_bytes; ne.promotion = promotion;
    const cuuint64_t eb = static_cast<cuuint64_t>(elem_bytes);
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(S),
                                static_cast<cuuint64_t>(H), static_cast<cuuint64_t>(B)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(ss) * eb, static_cast<cuuint64_t>(sh) * eb,
                                   static_cast<cuuint64_t>(sb) * eb};
    const cuuint32_t box[4] = {static_cast<cuuint32_t>(swizzle_bytes / elem_bytes), static_cast<cuuint32_t>(box_rows),
                              static_cast<cuuint32_t>(box_heads), 1u};
    const cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
    const CUresult r = h->encode(&ne.map, elem_bytes == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8,
                                 4, const_cast<void*>(ptr),
                                 dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 swizzle_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                                 static_cast<CUtensorMapL2promotion>(promotion),
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return FA_ERR_INVALID_ARG;     // strides or extents the TMA unit cannot express
    ne.stamp = ++h->stamp;
    if (static_cast<int>(h->maps.size()) < kMapCacheSize) {
        h->maps.push_back(ne);
        *out = &h->maps.back().map;
    } else {
        size_t victim = 0;
        for (size_t i = 1; i < h->maps.size(); ++i)
            if (h->maps[i].stamp < h->maps[victim].stamp) victim = i;
        h->maps[victim] = ne;
        *out = &h->maps[victim].map;
    }
    return FA_OK;
}

// Raises a kernel's dynamic shared-memory limit once per handle (the attribute is per device and
// function; the handle remembers which kernels it has prepared, by their address).
template <typename Kernel>
fa_status ensure_smem_attr(fa_handle* h, Kernel kernel, int bytes) {
    const void* key = reinterpret_cast<const void*>(kernel);
    for (const void* k : h->attr_done)
        if (k == key) return FA_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        cudaGetLastError();
        return FA_ERR_CUDA;
    }
    try {
        h->attr_done.push_back(key);
    } catch (...) {
        // (no memory to remember it in: the next call sets the limit again)
    }
    return FA_OK;
}

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Number of (batch, query head) instances scheduled together.  The K and V of a group (read again
// by every query tile of its heads) should fit in about a third of the 126 MB L2, a group holds
// whole GQA groups, and the groups are made equal in size: a small last group would start its
// longest items late and leave most SMs idle under them.
inline int heads_per_group(long long kv_bytes_per_head, int B, int Hq, int Hkv) {
    const long long budget = 48ll << 20;      // 32 to 96 MB measure the same within 2 %
    long long kv_heads = budget / kv_bytes_per_head;
    if (kv_heads < 1) kv_heads = 1;
    const long long gqa = Hq / Hkv;
    const long long n_kv = static_cast<long long>(B) * Hkv;       // K/V heads in the batch
    if (kv_heads > n_kv) kv_heads = n_kv;
    const long long n_groups = (n_kv + kv_heads - 1) / kv_heads;
    kv_heads = (n_kv + n_groups - 1) / n_groups;
    return static_cast<int>(kv_heads * gqa);
}

}  // namespace fa_host
