// Tables of up to BAGUA_MAX_WORKERS workers' buffers as kernel arguments, and the tiles of rows that a launch goes through.
#pragma once
#include "batch.hpp"
#include "elements.hpp"

namespace bagua {

// P buffers of every worker (nullptr throughout where the call has none of a kind).
template <int P>
struct Lists {
    const void* at[P][BAGUA_MAX_WORKERS];
    uint32_t rows[BAGUA_MAX_WORKERS];
    uint32_t first_tile[BAGUA_MAX_WORKERS];   // a tile: so many rows of one worker
};
static_assert(BAGUA_MAX_WORKERS == 32, "a worker for each lane of half a wave");

// The table with worker i in lane i: which worker has a tile is one comparison and a count of bits, and what belongs to it is read from
// its lane.  (From the arguments that is a chain of scalar loads, a new one for every worker that is passed over.)
template <int P>
struct LaneLists {
    uint32_t first_tile, rows;
    uint64_t at[P];
    __device__ __forceinline__ explicit LaneLists(const Lists<P>& ls)
    {
        const uint32_t i = threadIdx.x & (BAGUA_MAX_WORKERS - 1);
        first_tile = ls.first_tile[i];
        rows = ls.rows[i];
#pragma unroll
        for (int p = 0; p < P; ++p) at[p] = reinterpret_cast<uintptr_t>(ls.at[p][i]);
    }
    static __device__ __forceinline__ uint32_t lane(uint32_t v, uint32_t w) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), static_cast<int>(w))); }
    static __device__ __forceinline__ uint64_t lane(uint64_t v, uint32_t w)
    {
        return static_cast<uint64_t>(lane(static_cast<uint32_t>(v >> 32), w)) << 32 | lane(static_cast<uint32_t>(v), w);
    }
};

// A tile's rows: of one worker, from row t0 on; all of it wave-uniform.
template <int P>
struct ListTile {
    uint64_t at[P];
    uint32_t t0, rows;         // rows: that exist, one at least
    // tile: one that exists
    __device__ __forceinline__ ListTile(const LaneLists<P>& table, uint32_t tile, uint32_t of)
    {
        typedef LaneLists<P> T;
        // the last worker whose tiles begin at `tile` or before it (of workers without rows, which begin there too, the one behind them)
        const uint32_t w = static_cast<uint32_t>(__popc(static_cast<uint32_t>(__ballot(table.first_tile <= tile)))) - 1u;
        t0 = (tile - T::lane(table.first_tile, w)) * of;
        rows = min(of, T::lane(table.rows, w) - t0);
#pragma unroll
        for (int p = 0; p < P; ++p) at[p] = T::lane(table.at[p], w);
    }
    template <typename T>
    __device__ __forceinline__ T* ptr(int p) const { return table_ptr<T>(at[p]); }
};

// Cuts the workers' rows into tiles of `of` rows; the value: how many there are, or more than kMaxGrid.
template <int P>
inline uint64_t tiles_of(Lists<P>& ls, const size_t* rows, int k, uint32_t of)
{
    uint64_t tiles = 0;
    for (int w = 0; w < BAGUA_MAX_WORKERS; ++w) {
        // (a worker that is not there begins behind the last tile)
        ls.first_tile[w] = w < k ? static_cast<uint32_t>(tiles) : 0xffffffffu;
        ls.rows[w] = w < k ? static_cast<uint32_t>(rows[w]) : 0;
        if (w < k) tiles += (rows[w] + of - 1) / of;
        if (tiles > kMaxGrid) return tiles;
    }
    return tiles;
}

// Bytes from a matrix's first element to its last.
inline size_t rows_bytes(size_t rows, size_t ld, size_t columns, size_t element) { return rows ? ((rows - 1) * ld + columns) * element : 0; }
constexpr size_t kMostStride = static_cast<size_t>(1) << 40;

}  // namespace bagua
