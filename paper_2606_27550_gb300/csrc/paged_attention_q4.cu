// paged_attention_q4.cu -- tree attention over pages of 4 bits (paged_attention.cuh).
#include "paged_attention.cuh"

namespace tv {

TB_BOUNDS_COUNTER(bounds_violations_paged_attention_q4)

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_tree_attention_q4(const tb_bank *bank, const tb_requests *req, const tb_pages_q4 *pages,
                                             int layer, const void *plan, size_t plan_bytes, const void *q, int n_rows,
                                             int n_q_heads, float scale, float softcap, const float *slopes, void *out,
                                             float *lse, void *workspace, size_t workspace_bytes, tb_stream stream)
{
    const auto fill = [&](PagedArgs &a, int layer) -> const char * {
        const long long off = (long long)layer * pages->layer_stride;
        a.k_pages = static_cast<const uint8_t *>(pages->k) + off;
        a.v_pages = static_cast<const uint8_t *>(pages->v) + off;
        a.page_units = (uint32_t)(pages->page_stride / 16);
        a.head_stride = pages->head_stride;
        return pages->page_stride / 16 <= 0xffffffffll ? nullptr : "a page stride of 2^36 bytes or more";
    };
    return attend<true>(bank, req, pages, layer, plan, plan_bytes, q, n_rows, n_q_heads, scale, softcap, slopes, out,
                        lse, workspace, workspace_bytes, stream, "paged_tree_attention_q4", check_pages_q4, fill);
}
