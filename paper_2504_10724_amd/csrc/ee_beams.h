// ee_beams.h -- the choice of a beam search's next beams: what the kernels get, launchers.
#pragma once

#include "ee_internal.h"

constexpr int BEAM_MAX_BEAMS = 64, BEAM_MAX_KEEP = 128;
constexpr int BEAM_SLICE = 4096;     // logits of a workgroup; less where that makes no more than 1024 of them

// What a slice of a row's logits leaves: its maximum, sum of exp(z - maximum) in 64 bits, and a list of logits with their places in the row,
// in any order, the `keep` largest among them.
struct BeamParts {
    float*   top;                  // [rows][slices]
    double*  sum;                  // [rows][slices]
    int32_t* count;                // [rows][slices]: of the list
    float*   value;                // [rows][slices][room]
    int32_t* place;                // [rows][slices][room]
    int32_t  room;
};
size_t beam_parts(const ee_beam_config& c, char* ws, BeamParts* parts);    // its bytes

int launch_beam_select(const ee_beam_config& c, const void* logits, int64_t stride, const float* score, const uint8_t* done,
                       const ee_beam_choice& out, char* ws, hipStream_t s);
