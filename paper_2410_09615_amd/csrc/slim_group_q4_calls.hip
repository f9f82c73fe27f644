// The calls of the products with 4-bit weights that have a scale for each group of inputs: arguments are looked at here, and the kernels are chosen.
#include <hip/hip_runtime.h>

#include "slim_group_q4.h"

namespace slim {

int gq4_launch_act_backward(const void *dH, int64_t h_ld, const void *G, int64_t g_ld, const void *U, int64_t u_ld, int32_t m, int32_t n, void *dG,
                            int64_t dg_ld, void *dU, int64_t du_ld, int32_t dtype, hipStream_t st);
int gq4_launch_stream(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                      const int64_t (&y_ld)[3], int32_t dtype, hipStream_t st);
int gq4_launch_rows(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                    const int64_t (&y_ld)[3], int32_t dtype, void *workspace, hipStream_t st);
int gq4_launch_back(const slim_group_q4_layer *one, const slim_group_q4_layer *second, int shift, const void *dY, int64_t ld, const void *dY2, int64_t ld2, int32_t m, void *dX,
                    int64_t dx_ld, int32_t dtype, void *workspace, hipStream_t st);
void gq4_stream_plan(int n, int k, int m, bool gated, int32_t *out);
void gq4_rows_plan(int n, int k, int m, bool gated, int32_t *out);
void gq4_back_plan(int n, int k, int m, int terms, int32_t *out);
int64_t gq4_rows_workspace(int n, int k, int m, bool gated);
int64_t gq4_back_workspace(int n, int k, int m, int terms);

// The kernels address a tile's tokens by 32 bits from the first one on; with longer rows a call goes token by token.
constexpr int64_t kLongRow = 1 << 23;
// A launch has fewer than 2^32 threads: where the weights of so many rows are streamed 128 to each two blocks of rows, or to each of a gated pair.
constexpr int kMostRows = (1 << 30) - 2 * kGq4Rows;

// Both layers of a gated block: of one shape and group.
static int gq4_check_pair(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, int *shift)
{
    const int one = gq4_check(gate, shift), two = gq4_check(up, shift);
    if (one == SLIM_ERR_NULL || two == SLIM_ERR_NULL) return SLIM_ERR_NULL;
    if (one == SLIM_ERR_SHAPE || two == SLIM_ERR_SHAPE || gate->n != up->n || gate->k != up->k || gate->group != up->group) return SLIM_ERR_SHAPE;
    return one != SLIM_OK ? one : two;
}

static size_t gq4_need(int32_t n, int32_t k, int32_t m, int32_t call)
{
    int64_t most = 0;
    for (const int tokens : {(int)m, 1}) {                           // (one: of a call that goes token by token)
        int64_t b = 0;
        if (call == SLIM_GROUP_Q4_GEMM || call == SLIM_GROUP_Q4_GATED)
            b = gq4_streamed(n, k, tokens, call == SLIM_GROUP_Q4_GATED) ? 0 : gq4_rows_workspace(n, k, tokens, call == SLIM_GROUP_Q4_GATED);
        else
            b = gq4_back_workspace(n, k, tokens, call == SLIM_GROUP_Q4_GATED_BACKWARD ? 2 : 1);
        most = b > most ? b : most;
    }
    return (size_t)most;
}

static int gq4_check_room(int32_t n, int32_t k, int32_t m, int32_t call, const void *workspace, size_t bytes)
{
    const size_t need = gq4_need(n, k, m, call);
    if (need && workspace && !aligned16(workspace)) return SLIM_ERR_ALIGN;
    return need && (!workspace || bytes < need) ? SLIM_ERR_WORKSPACE : SLIM_OK;
}

static int gq4_forward(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                       const int64_t (&y_ld)[3], int32_t dtype, void *workspace, hipStream_t st)
{
    if (x_ld < kLongRow || m == 1) {
        if (gq4_streamed(layer->n, layer->k, m, up != nullptr)) return gq4_launch_stream(layer, up, shift, X, x_ld, m, y, y_ld, dtype, st);
        return gq4_launch_rows(layer, up, shift, X, x_ld, m, y, y_ld, dtype, workspace, st);
    }
    for (int t = 0; t < m; ++t) {
        void *one[3];
        for (int i = 0; i < 3; ++i) one[i] = y[i] ? static_cast<uint16_t *>(y[i]) + t * y_ld[i] : nullptr;
        const int rc = gq4_forward(layer, up, shift, static_cast<const uint16_t *>(X) + t * x_ld, x_ld, 1, one, y_ld, dtype, workspace, st);
        if (rc != SLIM_OK) return rc;
    }
    return SLIM_OK;
}

static int gq4_backward(const slim_group_q4_layer *one, const slim_group_q4_layer *second, int shift, const void *dY, int64_t ld, const void *dY2, int64_t ld2, int32_t m, void *dX,
                        int64_t dx_ld, int32_t dtype, void *workspace, hipStream_t st)
{
    if ((ld < kLongRow && ld2 < kLongRow) || m == 1) return gq4_launch_back(one, second, shift, dY, ld, dY2, ld2, m, dX, dx_ld, dtype, workspace, st);
    for (int t = 0; t < m; ++t) {
        const int rc = gq4_launch_back(one, second, shift, static_cast<const uint16_t *>(dY) + t * ld, ld, dY2 ? static_cast<const uint16_t *>(dY2) + t * ld2 : nullptr, ld2, 1,
                                       static_cast<uint16_t *>(dX) + t * dx_ld, dx_ld, dtype, workspace, st);
        if (rc != SLIM_OK) return rc;
    }
    return SLIM_OK;
}

}  // namespace slim

using namespace slim;

extern "C" int slim_group_q4_workspace(int32_t n, int32_t k, int32_t m, int32_t call, size_t *bytes)
{
    if (!bytes) return SLIM_ERR_NULL;
    if (slim_group_q4_sizes(n, k, 128, nullptr, nullptr, nullptr) != SLIM_OK || m < 1 || call < SLIM_GROUP_Q4_GEMM || call > SLIM_GROUP_Q4_GATED_BACKWARD) return SLIM_ERR_SHAPE;
    *bytes = gq4_need(n, k, m, call);
    return SLIM_OK;
}

// What a call would launch (no launch, no device access but for its number of compute units).
extern "C" int slim_group_q4_plan(int32_t n, int32_t k, int32_t m, int32_t call, int32_t *out)
{
    size_t need;
    if (!out) return SLIM_ERR_NULL;
    const int status = slim_group_q4_workspace(n, k, m, call, &need);
    if (status != SLIM_OK) return status;
    const bool gated = call == SLIM_GROUP_Q4_GATED;
    if (gated || call == SLIM_GROUP_Q4_GEMM) {
        out[0] = gq4_streamed(n, k, m, gated) ? 0 : 1;
        if (out[0] == 0)
            gq4_stream_plan(n, k, m, gated, out);
        else
            gq4_rows_plan(n, k, m, gated, out);
    } else {
        out[0] = 2;
        gq4_back_plan(n, k, m, call == SLIM_GROUP_Q4_GATED_BACKWARD ? 2 : 1, out);
    }
    return SLIM_OK;
}

extern "C" int slim_group_q4_gemm(const slim_group_q4_layer *layer, const void *X, int64_t x_ld, int32_t m, void *Y, int64_t y_ld, int32_t dtype, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    if (!X || !Y) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check(layer, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (layer->n > kMostRows || m < 1 || !half_dtype(dtype) || x_ld < layer->k || y_ld < layer->n) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(X, dtype) || !whole_elements(Y, dtype)) return SLIM_ERR_ALIGN;
    const int room = gq4_check_room(layer->n, layer->k, m, SLIM_GROUP_Q4_GEMM, workspace, workspace_bytes);
    if (room != SLIM_OK) return room;
    void *const y[3] = {Y, nullptr, nullptr};
    const int64_t y_lds[3] = {y_ld, 0, 0};
    return gq4_forward(layer, nullptr, shift, X, x_ld, m, y, y_lds, dtype, workspace, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gemm_t(const slim_group_q4_layer *layer, const void *dY, int64_t dy_ld, int32_t m, void *dX, int64_t dx_ld, int32_t dtype, void *workspace,
                                    size_t workspace_bytes, void *stream)
{
    if (!dY || !dX) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check(layer, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (m < 1 || !half_dtype(dtype) || dy_ld < layer->n || dx_ld < layer->k) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(dY, dtype) || !whole_elements(dX, dtype)) return SLIM_ERR_ALIGN;
    const int room = gq4_check_room(layer->n, layer->k, m, SLIM_GROUP_Q4_GEMM_T, workspace, workspace_bytes);
    if (room != SLIM_OK) return room;
    return gq4_backward(layer, nullptr, shift, dY, dy_ld, nullptr, 0, m, dX, dx_ld, dtype, workspace, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gated(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, const void *X, int64_t x_ld, int32_t m, void *H, int64_t h_ld,
                                   void *G, int64_t g_ld, void *U, int64_t u_ld, int32_t dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !H) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check_pair(gate, up, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (gate->n > kMostRows / 2 || m < 1 || !half_dtype(dtype) || x_ld < gate->k || h_ld < gate->n || (G && g_ld < gate->n) || (U && u_ld < gate->n)) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(X, dtype) || !whole_elements(H, dtype) || !whole_elements(G, dtype) || !whole_elements(U, dtype)) return SLIM_ERR_ALIGN;
    const int room = gq4_check_room(gate->n, gate->k, m, SLIM_GROUP_Q4_GATED, workspace, workspace_bytes);
    if (room != SLIM_OK) return room;
    void *const y[3] = {H, G, U};
    const int64_t y_lds[3] = {h_ld, g_ld, u_ld};
    return gq4_forward(gate, up, shift, X, x_ld, m, y, y_lds, dtype, workspace, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gated_backward(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, const void *dH, int64_t dh_ld, const void *G,
                                            int64_t g_ld, const void *U, int64_t u_ld, int32_t m, void *dG, int64_t dg_ld, void *dU, int64_t du_ld, void *dX,
                                            int64_t dx_ld, int32_t dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!dH || !G || !U || !dG || !dU || !dX) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check_pair(gate, up, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    const int n = gate->n;
    if (m < 1 || !half_dtype(dtype) || dh_ld < n || g_ld < n || u_ld < n || dg_ld < n || du_ld < n || dx_ld < gate->k || dG == dU) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK) return status;
    for (const void *p : {dH, G, U, (const void *)dG, (const void *)dU, (const void *)dX})
        if (!whole_elements(p, dtype)) return SLIM_ERR_ALIGN;
    const int room = gq4_check_room(n, gate->k, m, SLIM_GROUP_Q4_GATED_BACKWARD, workspace, workspace_bytes);
    if (room != SLIM_OK) return room;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int rc = gq4_launch_act_backward(dH, dh_ld, G, g_ld, U, u_ld, m, n, dG, dg_ld, dU, du_ld, dtype, st);
    return rc != SLIM_OK ? rc : gq4_backward(gate, up, shift, dG, dg_ld, dU, du_ld, m, dX, dx_ld, dtype, workspace, st);
}
