// Which logits rows predict which tokens: made by psattn_logprob_plan, read by the heads' kernels (psattn_logprob.hip, psattn_head.hip).
#pragma once
#include <cstddef>
#include <cstdint>

#include "psattn.h"

struct psattn_lp_plan {
    int32_t T = 0, n_samples = 0, n_resp = 0, n_rows = 0;
    int64_t n_items = 0;
    int device = -1;
    void* d_blob = nullptr;
    // device views into d_blob
    const int32_t* rows = nullptr;         // [n_rows]   logits rows that predict something, ascending
    const int32_t* row_desc = nullptr;     // [T]        -1: predicts nothing; j >= 0: row inside response j (predicts token row + 1);
                                           //            -2 - i: last prompt row of sample i (predicts the first token of each response)
    const int32_t* resp_first = nullptr;   // [n_resp]   first token of the response
    const int32_t* resp_len = nullptr;     // [n_resp]
    const int32_t* resp_prev = nullptr;    // [n_resp]   last prompt row of its sample, -1 if the prompt is empty
    const int32_t* samp_ptr = nullptr;     // [n_samples + 1] responses of sample i
    const int32_t* item_ptr = nullptr;     // [n_resp + 1] items of response j: a row and the token that it predicts, one after the other
};
