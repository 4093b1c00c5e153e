// Host-side checks and the launch that the operators' entry points share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "host.h"
#include "quasar.h"

namespace quasar {

inline bool valid_dtype(quasar_dtype d) { return d == QUASAR_F32 || d == QUASAR_BF16; }
inline int64_t dtype_size(quasar_dtype d) { return d == QUASAR_BF16 ? 2 : 4; }
inline bool valid_act(quasar_activation a) { return a >= QUASAR_ACT_NONE && a <= QUASAR_ACT_GELU; }
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The bytes of a strided matrix: `width` of them in each of `rows` rows that
// are `pitch` apart.
struct Bytes {
    uintptr_t at;
    size_t rows, width, pitch;

    Bytes(const void* p, int64_t rows_, int64_t cols, int64_t ld, int64_t size)
        : at(reinterpret_cast<uintptr_t>(p)), rows(p ? (size_t)rows_ : 0), width((size_t)(cols * size)),
          pitch((size_t)(ld * size))
    {
    }
    Bytes(const void* p, int64_t n, int64_t size) : Bytes(p, 1, n, n, size) {}
    size_t span() const { return rows == 0 || width == 0 ? 0 : (rows - 1) * pitch + width; }
    bool operator==(const Bytes& o) const
    {
        return at == o.at && rows == o.rows && width == o.width && (rows <= 1 || pitch == o.pitch);
    }
};

// Whether two matrices share a byte.  Columns of one buffer (the same pitch)
// lie between each other's without: decided by where they lie in its rows.
inline bool overlaps(const Bytes& a, const Bytes& b)
{
    const size_t na = a.span(), nb = b.span();
    if (na == 0 || nb == 0 || a.at >= b.at + nb || b.at >= a.at + na) return false;
    const size_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((b.rows > 1 && b.pitch != pitch) || a.width > pitch || b.width > pitch) return true;
    const size_t from = b.at >= a.at ? (b.at - a.at) % pitch : (pitch - (a.at - b.at) % pitch) % pitch;
    return from < a.width || from + b.width > pitch;
}

// Sizes a 2-D view may have: coordinates are 32-bit on the device, offsets 64.
inline bool valid_shape(int64_t rows, int64_t cols, int64_t ld)
{
    constexpr int64_t kMax = (int64_t(1) << 31) - 256;
    return rows >= 0 && cols >= 0 && rows <= kMax && cols <= kMax && ld >= cols &&
           ld <= (int64_t(1) << 36) && (rows == 0 || ld <= (int64_t(1) << 58) / rows);
}

// An operand's rows start at 16-byte boundaries (the rule of tiled copies).
inline bool valid_operand(const void* p, int64_t rows, int64_t cols, int64_t ld)
{
    return valid_shape(rows, cols, ld) && (rows == 0 || cols == 0 || (p && aligned(p, 16) && ld % 8 == 0));
}

// -- launches ------------------------------------------------------------------

// A programmatic dependent launch: every kernel started by it waits for the
// grid before it in the stream before it touches global memory, and only its
// prologue (barriers, tensor memory, tensor maps) runs earlier.
inline quasar_status launch(const void* fn, void* params, dim3 grid, int threads, int cluster, size_t smem,
                            quasar_stream_t stream)
{
    if (smem > 0) {  // (kernels with static shared memory take no dynamic)
        const quasar_status st = host_allow_smem(fn, smem);
        if (st != QUASAR_OK) return st;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    void* args[] = {params};
    return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? QUASAR_OK : QUASAR_ERR_CUDA;
}

// -- tensor maps ---------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

}  // namespace quasar
