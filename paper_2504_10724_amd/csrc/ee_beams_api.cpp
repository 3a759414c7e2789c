// ee_beams_api.cpp -- the C ABI of the beam search's choice: argument checks.
#include "ee_beams.h"

#include <algorithm>
#include <cstdlib>

static int check_beams(const ee_beam_config* c) {
    if (c->n_groups < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: negative count");
    if (c->beams < 1 || c->beams > BEAM_MAX_BEAMS || c->keep < 1 || c->keep > BEAM_MAX_KEEP)
        return ee_fail(EE_ERR_SHAPE, "ee_beam_select: beams must be 1 to 64, keep 1 to 128");
    if (c->vocab < 1 || c->vocab > 1 << 30) return ee_fail(EE_ERR_SHAPE, "ee_beam_select: vocab must be 1 to 2^30");
    if (c->dtype != EE_F32 && c->dtype != EE_BF16) return ee_fail(EE_ERR_DTYPE, "ee_beam_select: unknown dtype");
    if (c->end_token < -1 || c->end_token >= c->vocab) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: end_token outside the vocabulary");
    if ((int64_t)c->n_groups * c->beams * ((c->vocab + (int64_t)BEAM_SLICE - 1) / BEAM_SLICE) >= MOST_BLOCKS)
        return ee_fail(EE_ERR_SHAPE, "ee_beam_select: more slices than a launch holds");
    return EE_OK;
}

extern "C" {

size_t ee_beam_workspace(const ee_beam_config* c) {
    if (!c || check_beams(c) != EE_OK) return 0;
    return beam_parts(*c, nullptr, nullptr);
}

int ee_beam_select(const ee_beam_config* c, const void* dev_logits, int64_t row_stride, const float* dev_score, const uint8_t* dev_done,
                   const ee_beam_choice* out, void* dev_workspace, size_t workspace_bytes, void* stream) {
    if (!c || !out) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: null pointer");
    const int rc = check_beams(c);
    if (rc != EE_OK) return rc;
    if (dev_done && c->end_token < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: beams have ended, but there is no end_token");
    if (c->n_groups == 0) return EE_OK;
    if (!dev_logits || !dev_score || !out->dev_score || !out->dev_parent || !out->dev_token)
        return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: null pointer");
    const bool same = c->keep == c->beams;
    if (!same && (out->dev_score == dev_score || (dev_done && out->dev_done == dev_done)))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: results in place of the inputs need keep == beams");
    if ((uintptr_t)dev_logits % (c->dtype == EE_BF16 ? 2 : 4) != 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: logits are not aligned to their type");
    const size_t need = beam_parts(*c, nullptr, nullptr);
    if (need > 0 && !dev_workspace) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: null workspace");
    if (workspace_bytes < need) return ee_fail(EE_ERR_CAPACITY, "ee_beam_select: workspace smaller than ee_beam_workspace");
    if ((uintptr_t)dev_workspace % 256 != 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: workspace must be 256-byte aligned");
    // A request's workgroup writes its results while others read: what one of them reads, another may write only if both are the same request's.
    const size_t rows = (size_t)c->n_groups * c->beams, kept = (size_t)c->n_groups * c->keep;
    const Span read[] = {{dev_score, 4 * rows}, {dev_done, rows}};
    const Span made[] = {{out->dev_score, 4 * kept}, {out->dev_done, kept}, {out->dev_parent, 4 * kept}, {out->dev_token, 4 * kept}, {dev_workspace, need}};
    const size_t element = c->dtype == EE_BF16 ? 2 : 4;
    const int64_t last = (int64_t)(rows - 1) * row_stride;           // the last row's first element
    const Span logits{(const char*)dev_logits + std::min<int64_t>(last, 0) * (int64_t)element, (size_t)(std::abs(last) + c->vocab) * element};
    bool apart = !made[4].meets(logits);
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < 2; ++j) apart = apart && ((i == j && made[i].p == read[j].p) || !made[i].meets(read[j]));
        for (int j = 0; j < i; ++j) apart = apart && !made[i].meets(made[j]);
    }
    if (!apart) return ee_fail(EE_ERR_INVALID_ARG, "ee_beam_select: results, workspace and what is read share their memory");
    return launch_beam_select(*c, dev_logits, row_stride, dev_score, dev_done, *out, (char*)dev_workspace, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
