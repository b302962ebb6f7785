// Attention of a chunk of new tokens over the paged cache.
//
// The query heads that share a kv head are rows of one problem: row i * group + g of (sequence, kv head) is new token i, head
// kv_head * group + g.  A wave takes 32 rows.  It computes the scores transposed, S^T = K Q^T, so that a lane holds scores of
// one row only (row lane % 32; the two halves of the wave hold different keys): maximum and sum of the softmax stay in the
// lane but for one exchange between the halves, and the weights come out in the order in which the next product,
// O^T = V^T P^T, wants them.  Neither scores nor weights pass through LDS.
//
//   RW = 4, 8: waves of 32 rows share each tile of keys and values (chunks of a prompt).
//   KW > 1: one set of 32 rows, each wave takes every KW-th tile through its own stretch of LDS, without barriers, and the
//           waves' results are joined at the end (single tokens: the time is that of reading the cache).
// Either may split the keys over several blocks; a second kernel then joins the blocks' results in order.
//
// Measured (heads of 128, 32 query and 8 kv heads, 16 bits, unless said):
//   prompts, 2 chunks of up to 4096 tokens over 12301 more keys, RW = 8: 1265 to 1315 us, 1.00 to 1.04 PFLOP/s, where a library product of 8192^3
//     reaches 1.13; the matrix units are fed half the cycles and the softmax's arithmetic takes nearly as many, at a clock that
//     the power limit holds down;
//   64 single tokens over up to 8192 keys each, KW = 4: 225 us for 1.2 GB, 5.3 TB/s;
//   1 token over 131002 keys, 16 and 2 heads, KW = 4, split: 26 to 30 us and 5 us to join (134 MB, 27 us at a copy's rate);
//   1 token over 128 keys, 12 heads of 64: 6.9 us; 128 tokens of 32 bits: 10.7 us: the chain of lookup, load, product, join.
//   Heads of 136 to 256 do not fit the registers: 107 of a lane lie in scratch with KW = 4 (64 tokens over 8192 keys, 8 heads of 256, bf16
//     1.22 ms, 3.5 TB/s; one token 36 us), 34 with RW = 4 in 32 bits (94 TFLOP/s); RW = 4 in 16 bits reaches 590 TFLOP/s.
#include "clear_attend_device.h"

using namespace ckks;

static AttendSizes sizes(const ckks_clear_attend_t &p) {
    const ckks_clear_pages_t &g = p.pages;
    return {p.batch, p.heads, g.kv_heads, g.head_dim, g.page_size, g.dtype, p.flags, p.window, 2.0 * g.head_dim * clear_dtype_bytes(g.dtype), nullptr};
}

extern "C" {

uint64_t ckks_clear_attend_work_bytes(const ckks_clear_attend_t *p) {
    AttendPlan n;
    return p && plan_attend(sizes(*p), n) ? n.work_bytes : 0;
}

int ckks_clear_attend(const ckks_clear_attend_t *p, void *stream) {
    const char *who = "ckks_clear_attend";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_pages_t &g = p->pages;
    if (int rc = check_cache(who, g, p->batch)) return rc;
    const u32 e = clear_dtype_bytes(g.dtype);
    const Extent cache[2] = {extent(g.d_k, e, {{g.n_pages, g.k_stride[0]}, {g.kv_heads, g.k_stride[1]}, {g.page_size, g.k_stride[2]}, {g.head_dim, 1}}),
                             extent(g.d_v, e, {{g.n_pages, g.v_stride[0]}, {g.kv_heads, g.v_stride[1]}, {g.page_size, g.v_stride[2]}, {g.head_dim, 1}})};
    AttendPlan n;
    AttendArgs a{};
    const AttendCall call{g, p->d_q, p->d_out, p->d_lse, p->d_work, p->work_bytes, p->q_stride, p->out_stride, p->scale, cache, 2};
    if (int rc = prepare_attend(who, sizes(*p), call, n, a)) return rc;
    if (!n.splits) return CKKS_OK;
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_attend<float, PLAIN>(a, n, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_attend<f16, PLAIN>(a, n, st)
                                       : launch_attend<bf16, PLAIN>(a, n, st);
}

}  // extern "C"
