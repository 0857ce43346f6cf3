// Internal declarations of the cache with accumulated weights.
#pragma once
#include "sh_window.h"

// Records of a cache: strides in elements, slots next to each other.
struct MassRecords {
    float *mass;
    int32_t *positions;
    long long ss, hs;             // between sequences, between heads
};

struct EvictParams {
    char *k, *v, *ko, *vo;        // where rows come from and go to (the same cache, or another)
    long long ss, hs, ls;         // bytes between sequences, heads, slots
    long long oss, ohs, ols;
    MassRecords rec, out;
    const int32_t *lengths;
    int32_t *left;                // [sequences]: rows that are left
    int sequences, heads, slots, keep, recent, row_bytes;
    bool in_place;
    int most;                     // moves of a unit at most
    int *count;                   // workspace: [units] moves
    int2 *moves;                  // [units][most]: (to, from)
};
size_t sh_mass_evict_scratch(long long units, int most);
cudaError_t sh_launch_mass_evict(const EvictParams &p, cudaStream_t s);

// Single tokens: add the step's weights to the masses, from the scores and totals that the attention has left (where it has not done so).
cudaError_t sh_launch_mass_fold(const WindowParams &p, cudaStream_t s);
// Prompts: add the weights of the chunk's rows to the masses of the keys they see; the chunk is in the cache already.
cudaError_t sh_launch_mass_columns_f32(const WindowParams &p, int D, cudaStream_t s);
cudaError_t sh_launch_mass_columns_umma(const WindowParams &p, int dtype, int D, cudaStream_t s);      // f16 and bf16
size_t sh_mass_columns_scratch(int tokens, int sequences, int hk, int g, int slots);      // bytes of `part` that either wants
// as sh_window_error_take
cudaError_t sh_mass_error_take(int *code, cudaStream_t s);
