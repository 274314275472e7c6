// The driver's function that describes a tensor for TMA, looked up at the first use: the library is not linked against the driver.
#ifndef LVSPEC_TENSOR_MAP_H_
#define LVSPEC_TENSOR_MAP_H_

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

namespace lvspec {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Null if the driver does not have it.  (Contexts may be used by several host threads: whichever come first write the same.)
inline EncodeTiledFn encode_fn()
{
    static std::atomic<EncodeTiledFn> fn{nullptr};
    EncodeTiledFn f = fn.load(std::memory_order_relaxed);
    if (!f) {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        f = reinterpret_cast<EncodeTiledFn>(sym);
        fn.store(f, std::memory_order_relaxed);
    }
    return f;
}

}  // namespace lvspec

#endif  // LVSPEC_TENSOR_MAP_H_
