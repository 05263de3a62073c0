// Internal declarations of what goes on around a step's attention: its tables, and
// the verification of drafted tokens.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tr.h"
#include "tr_divide.h"

namespace tr {

struct PagesArgs {
    int32_t seqs;
    const int32_t* change;
    const int32_t* kv_len;
    int32_t* kv_out;           // [seqs], may be kv_len
    int32_t* table;
    int32_t table_width;
    int64_t table_stride;
    int32_t page_size;
    Divisor by_page;           // filled in by the launch
    int32_t pages;
    int32_t* ring;             // [pages]
    const int32_t* state;      // [2]
    int32_t* state_out;        // [2], may be state
    int32_t* q_start;          // [seqs + 1]
    int64_t rows;
    int64_t* slots;            // [rows] or nullptr
    int32_t* pos;              // [rows] or nullptr
    int32_t* short_of;
};

hipError_t launch_pages(const PagesArgs& a, hipStream_t s);

struct VerifyArgs {
    int64_t rows;
    int32_t vocab;
    const void* target;
    const void* draft;         // or nullptr
    int64_t ld_target, ld_draft;
    const int32_t* ids;
    int32_t seqs;
    const int32_t* q_start;    // [seqs + 1]
    const float* accept;       // [rows]
    const float* draw;         // [seqs]
    int32_t width;
    int32_t* tokens;           // [seqs, width]
    int32_t* accepted;
    int32_t* change;
    double* part;              // [seqs, kSlices, 2]
};

// Slices of a row that are summed up one by one.
constexpr int kSlices = 256;

hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t s);

}  // namespace tr
