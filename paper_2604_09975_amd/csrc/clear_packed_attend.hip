// Attention over pages of 8 bits.  The kernels are those of clear_attend.hip: codes are brought to the queries' type, exactly, on their
// way into LDS, and from there on nothing differs.
#include "clear_attend_device.h"

using namespace ckks;

static AttendSizes sizes(const ckks_clear_packed_attend_t &p) {
    const ckks_clear_packed_t &g = p.pages;
    return {p.batch, p.heads, g.kv_heads, g.head_dim, g.page_size, g.dtype, p.flags, p.window, 2.0 * (g.head_dim + packed_blocks(g.head_dim))};
}
template <class T>
static int launch_packed(const PackedAttendArgs &a, const AttendPlan &n, u32 format, hipStream_t st) {
    return format == CKKS_CLEAR_E4M3 ? launch_attend<T, E4M3>(a, n, st) : launch_attend<T, I8>(a, n, st);
}

extern "C" {

uint64_t ckks_clear_packed_attend_work_bytes(const ckks_clear_packed_attend_t *p) {
    AttendPlan n;
    return p && plan_attend(sizes(*p), n) ? n.work_bytes : 0;
}

int ckks_clear_packed_attend(const ckks_clear_packed_attend_t *p, void *stream) {
    const char *who = "ckks_clear_packed_attend";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_packed_t &g = p->pages;
    if (int rc = check_packed(who, g, p->batch)) return rc;
    const PackedPlaces places = packed_places(g);
    AttendPlan n;
    PackedAttendArgs a{};
    const ckks_clear_pages_t codes = as_pages(g, false);
    const AttendCall call{codes, p->d_q, p->d_out, p->d_lse, p->d_work, p->work_bytes, p->q_stride, p->out_stride, p->scale, places.at, 4};
    if (int rc = prepare_attend(who, sizes(*p), call, n, a)) return rc;
    if (!n.splits) return CKKS_OK;
    a.kz = g.d_k_power, a.vz = g.d_v_power;
    for (int i = 0; i < 3; ++i) a.kzs[i] = g.k_power_stride[i], a.vzs[i] = g.v_power_stride[i];
    if (!g.n_pages) {  // as the codes
        a.kz = a.vz = (const unsigned char *)p->d_q;
        for (int i = 0; i < 3; ++i) a.kzs[i] = a.vzs[i] = 0;
    }
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_packed<float>(a, n, g.format, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_packed<f16>(a, n, g.format, st)
                                       : launch_packed<bf16>(a, n, g.format, st);
}

}  // extern "C"
