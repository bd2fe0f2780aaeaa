// C-ABI entry points of libvgc: argument checking, plan construction, kernel dispatch.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "vgc_epilogue.h"
#include "vgc_internal.h"

namespace vgc {

static thread_local char g_err[512] = "";

void set_error(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
}

int hip_check(hipError_t e, const char* what) {
    if (e == hipSuccess) return VGC_OK;
    set_error("%s: %s", what, hipGetErrorString(e));
    return VGC_ERR_HIP;
}

// Validates the group list and counts tiles.  Returns a vgc_status.
struct GroupStats { uint64_t n_runs; uint32_t n_segs; uint32_t max_group_tiles; bool whole_tiles, whole_lines; uint64_t hash; };

static int check_groups(const vgc_group* groups, uint32_t n_groups, uint64_t n, uint64_t* n_tiles_out,
                        GroupStats* stats_out = nullptr) {
    if (!groups) { set_error("groups is NULL"); return VGC_ERR_NULL; }
    if (n == 0 || n_groups == 0) { set_error("n and n_groups must be positive"); return VGC_ERR_SIZE; }
    uint64_t off = 0, tiles = 0, runs = 0, segs = 0;
    uint64_t hash = 0xCBF29CE484222325ull ^ n_groups;       // FNV-1a over the sizes (offsets follow from them)
    uint32_t most = 0, ragged = 0, odd = 0;
    for (uint32_t k = 0; k < n_groups; ++k) {
        hash = (hash ^ groups[k].size) * 0x100000001B3ull;
        if (groups[k].size == 0) { set_error("group %u is empty", k); return VGC_ERR_SIZE; }
        if (groups[k].size > VGC_MAX_GROUP_SIZE) {
            set_error("group %u has %u elements; a 28-bit index holds at most 2^28", k, groups[k].size);
            return VGC_ERR_GROUP_TOO_LARGE;
        }
        if (groups[k].offset != off || groups[k].reserved != 0) {
            set_error("group %u starts at %llu, expected %llu: groups must tile [0, n) in order", k,
                      (unsigned long long)groups[k].offset, (unsigned long long)off);
            return VGC_ERR_SIZE;
        }
        off += groups[k].size;
        const uint64_t nt = (groups[k].size + kTile - 1) / kTile;
        tiles += nt;
        runs += (nt + kRunTiles - 1) / kRunTiles;
        segs += (nt + kSegTiles - 1) / kSegTiles;
        if (nt > most) most = (uint32_t)nt;
        ragged |= groups[k].size % kTile;
        odd |= (uint32_t)groups[k].offset % 4;               // (not whole 16-byte pieces of a float buffer)
    }
    if (off != n) {
        set_error("groups cover %llu elements, n = %llu", (unsigned long long)off, (unsigned long long)n);
        return VGC_ERR_SIZE;
    }
    if (tiles > 0x7FFFFFFFull) { set_error("too many tiles (%llu)", (unsigned long long)tiles); return VGC_ERR_SIZE; }
    if (n_tiles_out) *n_tiles_out = tiles;
    if (stats_out) { stats_out->n_runs = runs; stats_out->n_segs = (uint32_t)segs; stats_out->max_group_tiles = most; stats_out->whole_tiles = ragged == 0; stats_out->whole_lines = odd == 0; stats_out->hash = hash; }
    return VGC_OK;
}

// The run and segment tables sit after the tile table; their sizes are bounded through the tile and
// group counts, so the layout reserves the bound and the offsets depend on (n_tiles, n_groups) only.
static size_t plan_bytes_for(uint64_t n_tiles, uint32_t n_groups, size_t* groups_off, size_t* tiles_off,
                             size_t* runs_off = nullptr, size_t* segs_off = nullptr) {
    size_t off = sizeof(PlanHeader);
    if (groups_off) *groups_off = off;
    off = align_up(off + (size_t)n_groups * sizeof(PlanGroup), 256);
    if (tiles_off) *tiles_off = off;
    off = align_up(off + n_tiles * sizeof(PlanTile), 256);
    if (runs_off) *runs_off = off;
    off = align_up(off + (n_tiles / kRunTiles + n_groups) * sizeof(PlanRun), 256);
    if (segs_off) *segs_off = off;
    off = align_up(off + (n_tiles / kSegTiles + n_groups) * sizeof(PlanSeg), 256);
    return off;
}

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct PlanView { const PlanGroup* groups; const PlanTile* tiles; const PlanRun* runs; const PlanSeg* segs; };

static PlanCheck plan_check(const void* plan_dev, const GroupStats& gs) {
    return PlanCheck{static_cast<const PlanHeader*>(plan_dev), gs.hash};
}

static PlanView plan_view(const void* plan_dev, uint64_t n_tiles, uint32_t n_groups) {
    size_t go, to, ro, so;
    plan_bytes_for(n_tiles, n_groups, &go, &to, &ro, &so);
    const char* b = static_cast<const char*>(plan_dev);
    return PlanView{reinterpret_cast<const PlanGroup*>(b + go), reinterpret_cast<const PlanTile*>(b + to),
                    reinterpret_cast<const PlanRun*>(b + ro), reinterpret_cast<const PlanSeg*>(b + so)};
}

// Working memory of vgc_sqgrad_noalloc: one copy per GPU the library's code object is loaded on, held until the
// process ends.  In host code the array's name is only a handle for hipGetSymbolAddress; kernels and copies get
// the device address that call returns.
static __device__ __align__(256) unsigned char scratch[VGC_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
static void* g_scratch_ptr[kMaxDevices];          // device address of `scratch` on each GPU, once looked up
static std::mutex g_scratch_mutex;

// Device address of `scratch` on the current GPU (looked up on the first call on that GPU).
static int static_scratch(void** out) {
    int dev = -1;
    int rc = hip_check(hipGetDevice(&dev), "hipGetDevice");
    if (rc != VGC_OK) return rc;
    if (dev < 0 || dev >= kMaxDevices) { set_error("vgc_sqgrad_noalloc: device ordinal %d out of range", dev); return VGC_ERR_HIP; }
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        rc = hip_check(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)), "hipGetSymbolAddress(scratch)");
        if (rc != VGC_OK) return rc;
        if (!p) { set_error("vgc_sqgrad_noalloc: no device address for the static scratch"); return VGC_ERR_HIP; }
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return VGC_OK;
}

}  // namespace vgc

using namespace vgc;

extern "C" {

const char* vgc_last_error(void) { return g_err; }

uint32_t vgc_tile_size(void) { return kTile; }

uint64_t vgc_tile_count(const vgc_group* groups, uint32_t n_groups, uint64_t n) {
    uint64_t t = 0;
    return check_groups(groups, n_groups, n, &t) == VGC_OK ? t : 0;
}

size_t vgc_plan_bytes(const vgc_group* groups, uint32_t n_groups, uint64_t n) {
    uint64_t t = 0;
    if (check_groups(groups, n_groups, n, &t) != VGC_OK) return 0;
    return plan_bytes_for(t, n_groups, nullptr, nullptr);
}

size_t vgc_scratch_bytes(const vgc_group* groups, uint32_t n_groups, uint64_t n) {
    uint64_t t = 0;
    if (check_groups(groups, n_groups, n, &t) != VGC_OK) return 0;
    return scratch_layout(t, n_groups).total;
}

size_t vgc_scratch_bitmap_offset(const vgc_group* groups, uint32_t n_groups, uint64_t n) {
    uint64_t t = 0;
    if (check_groups(groups, n_groups, n, &t) != VGC_OK) return 0;
    return scratch_layout(t, n_groups).bitmap_off;
}

int vgc_plan_build(const vgc_group* groups, uint32_t n_groups, uint64_t n, void* plan_host, size_t plan_bytes) {
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (!plan_host) { set_error("plan_host is NULL"); return VGC_ERR_NULL; }
    size_t go, to, ro, so;
    const size_t need = plan_bytes_for(n_tiles, n_groups, &go, &to, &ro, &so);
    if (plan_bytes < need) { set_error("plan buffer has %zu bytes, %zu needed", plan_bytes, need); return VGC_ERR_SIZE; }
    char* b = static_cast<char*>(plan_host);
    memset(b, 0, need);
    PlanHeader* h = reinterpret_cast<PlanHeader*>(b);
    h->magic = kPlanMagic; h->n = n; h->n_tiles = n_tiles; h->n_groups = n_groups; h->tile = kTile;
    h->groups_off = go; h->tiles_off = to; h->runs_off = ro; h->n_runs = gs.n_runs;
    h->segs_off = so; h->n_segs = gs.n_segs; h->groups_hash = gs.hash;
    PlanGroup* G = reinterpret_cast<PlanGroup*>(b + go);
    PlanTile* T = reinterpret_cast<PlanTile*>(b + to);
    PlanRun* R = reinterpret_cast<PlanRun*>(b + ro);
    PlanSeg* S = reinterpret_cast<PlanSeg*>(b + so);
    uint64_t t = 0, rn = 0;
    uint32_t sn = 0;
    for (uint32_t k = 0; k < n_groups; ++k) {
        G[k].offset = groups[k].offset; G[k].size = groups[k].size; G[k].first_tile = (uint32_t)t;
        const uint32_t group_first_seg = sn;
        uint32_t in_group = 0;
        for (uint64_t start = 0; start < groups[k].size; start += kTile, ++t, ++in_group) {
            if (in_group % kSegTiles == 0) {
                S[sn].group = k; S[sn].first_tile = in_group; S[sn].seg_in_group = sn - group_first_seg;
                S[sn].group_first_seg = group_first_seg;
                ++sn;
            }
            if (in_group % kRunTiles == 0) { R[rn].group = k; R[rn].first_tile = in_group; ++rn; }
            T[t].group = k; T[t].start = (uint32_t)start; T[t].seg = sn - 1; T[t].run = (uint32_t)(rn - 1);
        }
    }
    return VGC_OK;
}

size_t vgc_sqgrad_workspace_bytes(int kind, int dtype, uint32_t B, uint32_t P, uint32_t J, uint32_t C) {
    return sqgrad_workspace_bytes(kind, dtype, B, P, J, C);
}

int vgc_sqgrad(int kind, int dtype, const void* X, const void* D, uint32_t B, uint32_t P, uint32_t J, uint32_t C,
               float c, float* g_out, float* s_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (kind != VGC_FC && kind != VGC_CONV) { set_error("vgc_sqgrad: unknown kind %d", kind); return VGC_ERR_DTYPE; }
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_sqgrad: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (!X || !D || !s_out) { set_error("vgc_sqgrad: X, D and s_out are required"); return VGC_ERR_NULL; }
    if (B == 0 || P == 0 || J == 0 || C == 0) { set_error("vgc_sqgrad: zero dimension"); return VGC_ERR_SIZE; }
    if (kind == VGC_FC && P != 1) { set_error("vgc_sqgrad: the FC form has P = 1"); return VGC_ERR_SIZE; }
    if (!aligned(X, 16) || !aligned(D, 16) || !aligned(s_out, 16) || (g_out && !aligned(g_out, 16))) {
        set_error("vgc_sqgrad: pointers must be 16-byte aligned");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c)) { set_error("vgc_sqgrad: c is not finite"); return VGC_ERR_PARAM; }
    if (workspace && !aligned(workspace, 16)) { set_error("vgc_sqgrad: workspace must be 16-byte aligned"); return VGC_ERR_ALIGN; }
    return launch_sqgrad(kind, dtype, X, D, B, P, J, C, c, g_out, s_out, workspace, workspace_bytes,
                         static_cast<hipStream_t>(stream));
}

int vgc_sqgrad_noalloc(int kind, int dtype, const void* X, const void* D, uint32_t B, uint32_t P, uint32_t J, uint32_t C,
                       float c, float* g_out, float* s_out, void* stream) {
    if (kind != VGC_FC && kind != VGC_CONV) { set_error("vgc_sqgrad_noalloc: unknown kind %d", kind); return VGC_ERR_DTYPE; }
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_sqgrad_noalloc: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (B == 0 || P == 0 || J == 0 || C == 0) { set_error("vgc_sqgrad_noalloc: zero dimension"); return VGC_ERR_SIZE; }
    const size_t need = sqgrad_workspace_bytes(kind, dtype, B, P, J, C);
    if (need > (size_t)VGC_NOALLOC_SCRATCH_BYTES) {
        set_error("vgc_sqgrad_noalloc: this shape wants %zu bytes of working memory, the static buffer has %zu; "
                  "call vgc_sqgrad with a workspace of the caller's", need, (size_t)VGC_NOALLOC_SCRATCH_BYTES);
        return VGC_ERR_SIZE;
    }
    void* ws = nullptr;
    const int rc = static_scratch(&ws);
    if (rc != VGC_OK) return rc;
    return vgc_sqgrad(kind, dtype, X, D, B, P, J, C, c, g_out, s_out, ws, (size_t)VGC_NOALLOC_SCRATCH_BYTES, stream);
}

// Validates a convolution's geometry; on success the output extent.
static int conv2d_geometry(int dtype, uint32_t B, uint32_t H, uint32_t W, uint32_t Cin, uint32_t C, uint32_t kh, uint32_t kw,
                           uint32_t sh, uint32_t sw, uint32_t ph, uint32_t pw, uint32_t* Ho, uint32_t* Wo) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_sqgrad_conv2d: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (B == 0 || H == 0 || W == 0 || Cin == 0 || C == 0 || kh == 0 || kw == 0 || sh == 0 || sw == 0) {
        set_error("vgc_sqgrad_conv2d: zero dimension");
        return VGC_ERR_SIZE;
    }
    if (ph >= kh || pw >= kw || (uint64_t)H + 2 * ph < kh || (uint64_t)W + 2 * pw < kw) {
        set_error("vgc_sqgrad_conv2d: need pad < kernel <= input + 2 pad");
        return VGC_ERR_SIZE;
    }
    if ((uint64_t)kh * kw * Cin > 0x7FFFFFFFull || (uint64_t)H * W > 0x7FFFFFFFull) { set_error("vgc_sqgrad_conv2d: shape too large"); return VGC_ERR_SIZE; }
    *Ho = (H + 2 * ph - kh) / sh + 1;
    *Wo = (W + 2 * pw - kw) / sw + 1;
    if (conv_stem_supported(dtype, Cin, C, kh, kw)) return VGC_OK;        // a first layer: few input channels, small kh kw Cin
    if (!conv2d_supported(dtype, H, W, Cin, C, *Ho * *Wo)) {
        set_error("vgc_sqgrad_conv2d: needs C a multiple of 16 bytes, Cin a multiple of 16 bytes or kh kw Cin <= 160, and "
                  "per-sample tensors below 2 GiB");
        return VGC_ERR_SIZE;
    }
    return VGC_OK;
}

size_t vgc_sqgrad_conv2d_workspace_bytes(int dtype, uint32_t B, uint32_t H, uint32_t W, uint32_t Cin, uint32_t C,
                                         uint32_t kh, uint32_t kw, uint32_t sh, uint32_t sw, uint32_t ph, uint32_t pw) {
    uint32_t Ho, Wo;
    if (conv2d_geometry(dtype, B, H, W, Cin, C, kh, kw, sh, sw, ph, pw, &Ho, &Wo) != VGC_OK) return 0;
    const uint32_t J = kh * kw * Cin;
    if (conv_stem_supported(dtype, Cin, C, kh, kw)) return conv_stem_workspace_bytes(dtype, B, Ho * Wo, J, C);
    if (dtype == VGC_BF16) {
        // the larger of what the two kernels that may serve the layer want (which one runs depends on whether g is asked for)
        size_t need = conv_workspace_bytes(B, Ho * Wo, J, C);
        if (conv_taps_supported(H, W, Cin, C, kh, kw, sh, sw, ph, pw)) {
            const size_t t = conv_taps_workspace_bytes(B, Ho * Wo, Cin, C);
            if (t > need) need = t;
        }
        return need;
    }
    return conv_f32_workspace_bytes(B, Ho * Wo, J, C);
}

// Argument checks of vgc_sqgrad_conv2d; the output size on success.
static int conv2d_check(int dtype, const void* act, const void* D, uint32_t B, uint32_t H, uint32_t W, uint32_t Cin,
                        uint32_t C, uint32_t kh, uint32_t kw, uint32_t sh, uint32_t sw, uint32_t ph, uint32_t pw,
                        float c, const float* g_out, const float* s_out, const void* workspace, size_t workspace_bytes,
                        uint32_t* Ho, uint32_t* Wo) {
    if (!act || !D || !s_out) { set_error("vgc_sqgrad_conv2d: act, D and s_out are required"); return VGC_ERR_NULL; }
    int rc = conv2d_geometry(dtype, B, H, W, Cin, C, kh, kw, sh, sw, ph, pw, Ho, Wo);
    if (rc != VGC_OK) return rc;
    if (!aligned(act, 16) || !aligned(D, 16) || !aligned(s_out, 16) || (g_out && !aligned(g_out, 16)) ||
        (workspace && !aligned(workspace, 16))) {
        set_error("vgc_sqgrad_conv2d: pointers must be 16-byte aligned");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c)) { set_error("vgc_sqgrad_conv2d: c is not finite"); return VGC_ERR_PARAM; }
    if (conv_stem_supported(dtype, Cin, C, kh, kw) &&
        (!workspace || workspace_bytes < conv_stem_workspace_bytes(dtype, B, *Ho * *Wo, kh * kw * Cin, C))) {
        set_error("vgc_sqgrad_conv2d: a layer whose input channels are not a multiple of 16 bytes needs the workspace "
                  "vgc_sqgrad_conv2d_workspace_bytes() asks for");
        return VGC_ERR_SIZE;
    }
    return VGC_OK;
}

int vgc_sqgrad_conv2d(int dtype, const void* act, const void* D, uint32_t B, uint32_t H, uint32_t W, uint32_t Cin,
                      uint32_t C, uint32_t kh, uint32_t kw, uint32_t sh, uint32_t sw, uint32_t ph, uint32_t pw,
                      float c, float* g_out, float* s_out, void* workspace, size_t workspace_bytes, void* stream) {
    uint32_t Ho, Wo;
    const int rc = conv2d_check(dtype, act, D, B, H, W, Cin, C, kh, kw, sh, sw, ph, pw, c, g_out, s_out, workspace, workspace_bytes, &Ho, &Wo);
    if (rc != VGC_OK) return rc;
    return launch_conv2d(dtype, act, D, B, H, W, Cin, C, kh, kw, sh, sw, ph, pw, Ho, Wo, c, g_out, s_out, workspace, workspace_bytes,
                         static_cast<hipStream_t>(stream));
}

// The library's own streams for vgc_sqgrad_conv2d_batch: one set per device, made on first use (default priority).
namespace {
constexpr int kSideStreams = 4;
struct SideStreams {
    bool ready = false;
    hipStream_t s[kSideStreams];
    hipEvent_t fork, join[kSideStreams];
};
std::mutex g_side_mutex;                                  // one batch call submits at a time per process
SideStreams g_side[64];
}  // namespace

int vgc_sqgrad_conv2d_batch(const vgc_conv2d_layer* layers, uint32_t n_layers, void* stream) {
    if (!layers && n_layers) { set_error("vgc_sqgrad_conv2d_batch: layers is NULL"); return VGC_ERR_NULL; }
    std::vector<uint32_t> Ho(n_layers), Wo(n_layers);
    for (uint32_t k = 0; k < n_layers; ++k) {             // every layer is checked before anything is launched
        const vgc_conv2d_layer& L = layers[k];
        const int rc = conv2d_check(L.dtype, L.act, L.D, L.B, L.H, L.W, L.Cin, L.C, L.kh, L.kw, L.stride_h, L.stride_w, L.pad_h,
                                    L.pad_w, L.c, L.g_out, L.s_out, L.workspace, L.workspace_bytes, &Ho[k], &Wo[k]);
        if (rc != VGC_OK) return rc;
    }
    hipStream_t user = static_cast<hipStream_t>(stream);
    int dev = 0;
    int rc = hip_check(hipGetDevice(&dev), "hipGetDevice");
    if (rc != VGC_OK) return rc;
    if (dev < 0 || dev >= 64) { set_error("vgc_sqgrad_conv2d_batch: device %d out of range", dev); return VGC_ERR_PARAM; }
    std::lock_guard<std::mutex> lock(g_side_mutex);
    SideStreams& S = g_side[dev];
    if (!S.ready) {
        for (int i = 0; i < kSideStreams; ++i) {
            if ((rc = hip_check(hipStreamCreateWithFlags(&S.s[i], hipStreamNonBlocking), "hipStreamCreate")) != VGC_OK) return rc;
            if ((rc = hip_check(hipEventCreateWithFlags(&S.join[i], hipEventDisableTiming), "hipEventCreate")) != VGC_OK) return rc;
        }
        if ((rc = hip_check(hipEventCreateWithFlags(&S.fork, hipEventDisableTiming), "hipEventCreate")) != VGC_OK) return rc;
        S.ready = true;
    }
    // Which stream takes which layer.  A layer of 2e10 multiply-adds or more fills the chip by itself; it stays on the
    // caller's stream.  Of the others each goes to the least loaded side stream.  What the rule costs and gives: the 53
    // small layers of ResNet-50 take 2.92 ms on one stream and 2.30 so (2.24 when the caller spreads all layers over four
    // streams); VGG-16, most of whose layers are above the line, 2.25 and 2.23 (2.18).  Spreading the large ones too took
    // between 1.7 % more and 2.5 % less on VGG-16 in eight comparisons, 0.3 % less on average.
    std::vector<int> lane_of(n_layers, 0);
    double load[kSideStreams + 1] = {0.0};               // multiply-adds queued on each stream so far
    bool lane_used[kSideStreams + 1] = {false};
    uint32_t n_small = 0;
    for (uint32_t k = 0; k < n_layers; ++k) {
        const vgc_conv2d_layer& L = layers[k];
        const double macs = (double)L.B * Ho[k] * Wo[k] * L.kh * L.kw * L.Cin * L.C;
        if (macs < 2e10) ++n_small;
    }
    for (uint32_t k = 0; k < n_layers; ++k) {
        const vgc_conv2d_layer& L = layers[k];
        const double macs = (double)L.B * Ho[k] * Wo[k] * L.kh * L.kw * L.Cin * L.C;
        int lane = 0;
        if (n_small > 1 && macs < 2e10) {
            lane = 1;
            for (int i = 2; i <= kSideStreams; ++i)
                if (load[i] < load[lane]) lane = i;
        }
        load[lane] += macs + 2e8;                        // (+ a launch's worth)
        lane_of[k] = lane;
        lane_used[lane] = true;
    }
    // fork: the side streams that get work start after whatever the caller's stream holds so far
    bool forked = false;
    for (int i = 1; i <= kSideStreams; ++i) {
        if (!lane_used[i]) continue;
        if (!forked && (rc = hip_check(hipEventRecord(S.fork, user), "hipEventRecord")) != VGC_OK) return rc;
        forked = true;
        if ((rc = hip_check(hipStreamWaitEvent(S.s[i - 1], S.fork, 0), "hipStreamWaitEvent")) != VGC_OK) return rc;
    }
    int first_error = VGC_OK;
    for (uint32_t k = 0; k < n_layers; ++k) {
        const vgc_conv2d_layer& L = layers[k];
        hipStream_t st = lane_of[k] == 0 ? user : S.s[lane_of[k] - 1];
        const int r = launch_conv2d(L.dtype, L.act, L.D, L.B, L.H, L.W, L.Cin, L.C, L.kh, L.kw, L.stride_h, L.stride_w, L.pad_h,
                                    L.pad_w, Ho[k], Wo[k], L.c, L.g_out, L.s_out, L.workspace, L.workspace_bytes, st);
        if (r != VGC_OK && first_error == VGC_OK) first_error = r;
    }
    // join: the caller's stream continues when every side stream is done (also after a failed launch)
    for (int i = 1; i <= kSideStreams; ++i) {
        if (!lane_used[i]) continue;
        if ((rc = hip_check(hipEventRecord(S.join[i - 1], S.s[i - 1]), "hipEventRecord")) != VGC_OK) return rc;
        if ((rc = hip_check(hipStreamWaitEvent(user, S.join[i - 1], 0), "hipStreamWaitEvent")) != VGC_OK) return rc;
    }
    return first_error;
}

// first_group, group_count: the groups the launch covers (all of them for the whole-model calls)
static int accumulate_select_any(const float* g, const float* s, float* r, float* v, uint64_t n,
                                 const vgc_group* groups, uint32_t n_groups, const void* plan,
                                 uint32_t first_group, uint32_t group_count,
                                 float alpha, float zeta, float tau, bool hybrid, void* scratch, void* stream) {
    if (!g || !s || !r || !v || !plan || !scratch) { set_error("vgc_accumulate_select: NULL pointer"); return VGC_ERR_NULL; }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (first_group > n_groups || group_count > n_groups - first_group) {
        set_error("vgc_accumulate_select_range: groups %u .. %u + %u are not inside the list of %u", first_group, first_group, group_count, n_groups);
        return VGC_ERR_SIZE;
    }
    if (!aligned(g, 4) || !aligned(s, 4) || !aligned(r, 4) || !aligned(v, 4) || !aligned(plan, 256) || !aligned(scratch, 256)) {
        set_error("vgc_accumulate_select: g, s, r, v need 4-byte, plan and scratch 256-byte alignment");
        return VGC_ERR_ALIGN;
    }
    if (!(alpha >= 0.0f) || !std::isfinite(alpha) || !(zeta > 0.0f) || !(zeta <= 1.0f)) {
        set_error("vgc_accumulate_select: need alpha >= 0 finite and 0 < zeta <= 1 (got %g, %g)", alpha, zeta);
        return VGC_ERR_PARAM;
    }
    if (hybrid && (!(tau >= 0.0f) || !std::isfinite(tau))) {
        set_error("vgc_accumulate_select_hybrid: need tau >= 0 finite (got %g)", tau);
        return VGC_ERR_PARAM;
    }
    uint64_t tile0 = 0, tiles = 0;
    for (uint32_t k = 0; k < first_group + group_count; ++k) {
        const uint64_t nt = (groups[k].size + kTile - 1) / kTile;
        if (k < first_group) tile0 += nt; else tiles += nt;
    }
    const ScratchLayout L = scratch_layout(n_tiles, n_groups);
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    char* sc = static_cast<char*>(scratch);
    const bool vec = aligned(g, 16) && aligned(s, 16) && aligned(r, 16) && aligned(v, 16);
    return launch_accumulate_select(plan_check(plan, gs), reinterpret_cast<uint32_t*>(sc + L.flags_off), g, s, r, v, pv.groups, pv.tiles,
                                    tile0, tiles,
                                    reinterpret_cast<TileHdr*>(sc + L.tile_hdr_off),
                                    reinterpret_cast<uint32_t*>(sc + L.bitmap_off),
                                    reinterpret_cast<uint16_t*>(sc + L.staging_off),
                                    alpha, zeta, tau, hybrid, vec, static_cast<hipStream_t>(stream));
}

int vgc_accumulate_select(const float* g, const float* s, float* r, float* v, uint64_t n,
                          const vgc_group* groups, uint32_t n_groups, const void* plan,
                          float alpha, float zeta, void* scratch, void* stream) {
    return accumulate_select_any(g, s, r, v, n, groups, n_groups, plan, 0, n_groups, alpha, zeta, 0.0f, false, scratch, stream);
}

int vgc_accumulate_select_hybrid(const float* g, const float* s, float* r, float* v, uint64_t n,
                                 const vgc_group* groups, uint32_t n_groups, const void* plan,
                                 float alpha, float zeta, float tau, void* scratch, void* stream) {
    return accumulate_select_any(g, s, r, v, n, groups, n_groups, plan, 0, n_groups, alpha, zeta, tau, true, scratch, stream);
}

int vgc_accumulate_select_range(const float* g, const float* s, float* r, float* v, uint64_t n,
                                const vgc_group* groups, uint32_t n_groups, const void* plan,
                                uint32_t first_group, uint32_t group_count,
                                float alpha, float zeta, void* scratch, void* stream) {
    return accumulate_select_any(g, s, r, v, n, groups, n_groups, plan, first_group, group_count, alpha, zeta, 0.0f, false, scratch, stream);
}

size_t vgc_sqgrad_accumulate_select_workspace_bytes(int dtype, uint32_t B, uint32_t J, uint32_t C) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) return 0;
    return fused_fc_workspace_bytes(dtype, B, J, C);
}

int vgc_sqgrad_accumulate_select(int dtype, const void* X, const void* D, uint32_t B, uint32_t J, uint32_t C, float c,
                                 float* r, float* v, uint64_t n, const vgc_group* groups, uint32_t n_groups, const void* plan,
                                 uint32_t group, float alpha, float zeta, void* scratch, void* workspace, size_t workspace_bytes,
                                 float* g_out, float* s_out, void* stream) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_sqgrad_accumulate_select: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (!X || !D || !r || !v || !plan || !scratch || !workspace) { set_error("vgc_sqgrad_accumulate_select: NULL pointer"); return VGC_ERR_NULL; }
    if ((g_out == nullptr) != (s_out == nullptr)) { set_error("vgc_sqgrad_accumulate_select: g_out and s_out go together"); return VGC_ERR_NULL; }
    if (B == 0 || J == 0 || C == 0) { set_error("vgc_sqgrad_accumulate_select: zero dimension"); return VGC_ERR_SIZE; }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (group >= n_groups || (uint64_t)J * C != groups[group].size) {
        set_error("vgc_sqgrad_accumulate_select: group %u does not exist or does not have J x C = %llu elements", group,
                  (unsigned long long)J * C);
        return VGC_ERR_SIZE;
    }
    const size_t need = fused_fc_workspace_bytes(dtype, B, J, C);
    if (need == 0) {
        set_error("vgc_sqgrad_accumulate_select: C = %u is neither a multiple of 2048 nor 256, 512 or 1024 "
                  "(use vgc_sqgrad and vgc_accumulate_select)", C);
        return VGC_ERR_SIZE;
    }
    if (workspace_bytes < need) { set_error("vgc_sqgrad_accumulate_select: workspace has %zu bytes, %zu needed", workspace_bytes, need); return VGC_ERR_SIZE; }
    const size_t es = dtype == VGC_BF16 ? 2 : 4;
    if (!aligned(X, es) || !aligned(D, es) || !aligned(r, 4) || !aligned(v, 4) || !aligned(plan, 256) || !aligned(scratch, 256) ||
        !aligned(workspace, 16) || !aligned(g_out, 4) || !aligned(s_out, 4)) {
        set_error("vgc_sqgrad_accumulate_select: misaligned pointer");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c) || !(alpha >= 0.0f) || !std::isfinite(alpha) || !(zeta > 0.0f) || !(zeta <= 1.0f)) {
        set_error("vgc_sqgrad_accumulate_select: need c finite, alpha >= 0 finite and 0 < zeta <= 1");
        return VGC_ERR_PARAM;
    }
    const ScratchLayout L = scratch_layout(n_tiles, n_groups);
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    char* sc = static_cast<char*>(scratch);
    return launch_fused_fc_select(plan_check(plan, gs), reinterpret_cast<uint32_t*>(sc + L.flags_off), dtype, X, D, B, J, C, c, r, v,
                                  pv.groups, group, reinterpret_cast<TileHdr*>(sc + L.tile_hdr_off),
                                  reinterpret_cast<uint32_t*>(sc + L.bitmap_off), reinterpret_cast<uint16_t*>(sc + L.staging_off),
                                  alpha, zeta, workspace, g_out, s_out, static_cast<hipStream_t>(stream));
}

int vgc_pack(uint64_t n, const vgc_group* groups, uint32_t n_groups, const void* plan, void* scratch,
             uint32_t* words_out, uint64_t words_cap, vgc_group_hdr* hdrs_out,
             vgc_pack_status* status_out, void* stream) {
    if (!plan || !scratch || !hdrs_out || !status_out || (!words_out && words_cap)) {
        set_error("vgc_pack: NULL pointer");
        return VGC_ERR_NULL;
    }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (!aligned(plan, 256) || !aligned(scratch, 256) || !aligned(words_out, 4) || !aligned(hdrs_out, 8) || !aligned(status_out, 8)) {
        set_error("vgc_pack: misaligned pointer");
        return VGC_ERR_ALIGN;
    }
    const ScratchLayout L = scratch_layout(n_tiles, n_groups);
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    char* sc = static_cast<char*>(scratch);
    return launch_pack(plan_check(plan, gs), reinterpret_cast<const uint32_t*>(sc + L.flags_off), pv.groups, pv.tiles, pv.segs, n_tiles, n_groups, gs.n_segs, gs.max_group_tiles,
                       reinterpret_cast<TileHdr*>(sc + L.tile_hdr_off),
                       reinterpret_cast<SegTmp*>(sc + L.seg_tmp_off),
                       reinterpret_cast<const uint16_t*>(sc + L.staging_off),
                       words_out, words_cap, hdrs_out, status_out, static_cast<hipStream_t>(stream));
}

uint64_t vgc_run_count(const vgc_group* groups, uint32_t n_groups, uint64_t n) {
    uint64_t t = 0;
    GroupStats gs;
    return check_groups(groups, n_groups, n, &t, &gs) == VGC_OK ? gs.n_runs : 0;
}

int vgc_pack_compact(uint64_t n, const vgc_group* groups, uint32_t n_groups, const void* plan, void* scratch,
                     uint8_t* stream_out, uint64_t stream_cap, uint16_t* tile_bytes_out, uint64_t* run_offsets_out,
                     vgc_group_hdr* hdrs_out, vgc_pack_status* status_out, void* stream) {
    if (!plan || !scratch || !hdrs_out || !status_out || !tile_bytes_out || !run_offsets_out || (!stream_out && stream_cap)) {
        set_error("vgc_pack_compact: NULL pointer");
        return VGC_ERR_NULL;
    }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (!aligned(plan, 256) || !aligned(scratch, 256) || !aligned(tile_bytes_out, 2) || !aligned(run_offsets_out, 8) ||
        !aligned(hdrs_out, 8) || !aligned(status_out, 8)) {
        set_error("vgc_pack_compact: misaligned pointer");
        return VGC_ERR_ALIGN;
    }
    const ScratchLayout L = scratch_layout(n_tiles, n_groups);
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    char* sc = static_cast<char*>(scratch);
    const PlanCheck pc = plan_check(plan, gs);
    return launch_pack_compact(pc, reinterpret_cast<const uint32_t*>(sc + L.flags_off), pv.groups, pv.tiles, pv.runs, pv.segs, n_tiles,
                               gs.n_runs, n_groups, gs.n_segs, gs.max_group_tiles, reinterpret_cast<TileHdr*>(sc + L.tile_hdr_off),
                               reinterpret_cast<SegTmp*>(sc + L.seg_tmp_off), reinterpret_cast<const uint16_t*>(sc + L.staging_off),
                               stream_out, stream_cap, tile_bytes_out, run_offsets_out, hdrs_out, status_out,
                               static_cast<hipStream_t>(stream));
}

// The batched decoders with the tiles of a wave given (a power of two up to a run's 64, 0: by the rule).  Not part of the
// interface: the public calls below pass 0; tests run on small parameter sets what only large ones lead to.
static bool tiles_ok(uint32_t tiles_per_wave) {
    if (tiles_per_wave <= kRunTiles && (tiles_per_wave & (tiles_per_wave - 1u)) == 0) return true;
    set_error("tiles_per_wave = %u is neither 0 nor a power of two up to %u", tiles_per_wave, kRunTiles);
    return false;
}

int vgc_tiles_unpack_compact_add_batch(const uint8_t* const* streams, const uint64_t* stream_bytes, const uint16_t* const* tile_bytes,
                                       const uint64_t* const* run_offsets, const vgc_group_hdr* const* hdrs, uint32_t p,
                                       const vgc_group* groups, uint32_t n_groups, const void* plan, float scale, int overwrite,
                                       float* dense_out, uint64_t n, void* stream, uint32_t tiles_per_wave) {
    if (!tiles_ok(tiles_per_wave)) return VGC_ERR_PARAM;
    if (!plan || !dense_out || (p && (!streams || !stream_bytes || !tile_bytes || !run_offsets || !hdrs))) {
        set_error("vgc_unpack_compact_add_batch: NULL pointer");
        return VGC_ERR_NULL;
    }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    for (uint32_t w = 0; w < p; ++w) {
        if (!hdrs[w] || !tile_bytes[w] || !run_offsets[w] || (!streams[w] && stream_bytes[w])) {
            set_error("vgc_unpack_compact_add_batch: message %u has a NULL pointer", w);
            return VGC_ERR_NULL;
        }
        if (!aligned(tile_bytes[w], 2) || !aligned(run_offsets[w], 8) || !aligned(hdrs[w], 8)) {
            set_error("vgc_unpack_compact_add_batch: message %u is misaligned", w);
            return VGC_ERR_ALIGN;
        }
    }
    if (!aligned(plan, 256) || !aligned(dense_out, 4)) { set_error("vgc_unpack_compact_add_batch: misaligned pointer"); return VGC_ERR_ALIGN; }
    if (!std::isfinite(scale)) { set_error("vgc_unpack_compact_add_batch: scale is not finite"); return VGC_ERR_PARAM; }
    if (p == 0 && !overwrite) return VGC_OK;
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    return launch_unpack_compact_batch(plan_check(plan, gs), streams, stream_bytes, tile_bytes, run_offsets, hdrs, p, pv.groups, pv.runs,
                                       n_tiles, gs.n_runs, scale, overwrite, dense_out, tiles_per_wave, static_cast<hipStream_t>(stream));
}

int vgc_unpack_compact_add_batch(const uint8_t* const* streams, const uint64_t* stream_bytes, const uint16_t* const* tile_bytes,
                                 const uint64_t* const* run_offsets, const vgc_group_hdr* const* hdrs, uint32_t p,
                                 const vgc_group* groups, uint32_t n_groups, const void* plan, float scale, int overwrite,
                                 float* dense_out, uint64_t n, void* stream) {
    return vgc_tiles_unpack_compact_add_batch(streams, stream_bytes, tile_bytes, run_offsets, hdrs, p, groups, n_groups, plan, scale,
                                              overwrite, dense_out, n, stream, 0);
}

int vgc_unpack_add(const uint32_t* words, uint64_t n_words, const vgc_group_hdr* hdrs,
                   const vgc_group* groups, uint32_t n_groups, const void* plan,
                   float scale, float* dense_out, uint64_t n, void* stream) {
    if (!hdrs || !plan || !dense_out || (!words && n_words)) { set_error("vgc_unpack_add: NULL pointer"); return VGC_ERR_NULL; }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    if (!aligned(plan, 256) || !aligned(words, 4) || !aligned(hdrs, 8) || !aligned(dense_out, 4)) {
        set_error("vgc_unpack_add: misaligned pointer");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(scale)) { set_error("vgc_unpack_add: scale is not finite"); return VGC_ERR_PARAM; }
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    // A message that touches most cache lines of the buffer anyway (going by n_words) is decoded tile by tile like a
    // batch of one: the same additions, the buffer streamed once instead of read and written line by line under 64
    // scattered lanes.  The line is an eighth of the elements, and from twice the last-level cache on (512 MB), where the
    // scattered lines come from memory also when the buffer has just been written, a sixteenth, or a twelfth where groups begin
    // anywhere and tiles are read in pieces of lines.  By words / by tiles, us, on a buffer just written (on a cold one):
    // 25 M parameters 37 / 43 (45 / 47) at 6.5 %, 43 / 43 (47 / 47) at 10 %; 75 M 89 / 107 (112 / 114) and 108 / 108 (119 / 115);
    // 138 M 173 / 191 (158 / 198) at 4 %, 223 / 191 (201 / 206) at 6.5 %, 231 / 192 (210 / 209) at 8 %; 400 M 507 / 531 (485 / 552)
    // at 4 %, 630 / 541 (604 / 575) at 6.5 %, 685 / 542 (675 / 598) at 10 %.  With groups that begin anywhere 138 M 214 / 218
    // (201 / 214) at 6.25 %, 225 / 219 (210 / 214) at 7.5 %, 232 / 222 (218 / 217) at 9 %; 268 M 421 / 436 (402 / 431), 439 / 441
    // (420 / 436), 454 / 448 (438 / 440).
    const bool whole = gs.whole_lines && aligned(dense_out, 16);
    const uint64_t dense_words = n < (1ull << 27) ? n / 8 : whole ? n / 16 : n / 12;
    if (n_words && n_words >= dense_words) {
        const uint32_t* const wl[1] = {words};
        const uint64_t nl[1] = {n_words};
        const vgc_group_hdr* const hl[1] = {hdrs};
        return launch_unpack_add_batch(plan_check(plan, gs), wl, nl, hl, 1, pv.groups, pv.tiles, pv.runs, n_tiles, gs.n_runs, gs.whole_tiles, scale, 0, dense_out, 0,
                                       static_cast<hipStream_t>(stream));
    }
    return launch_unpack_add(plan_check(plan, gs), words, n_words, hdrs, pv.groups, n_groups, scale, dense_out, static_cast<hipStream_t>(stream));
}

int vgc_tiles_unpack_add_batch(const uint32_t* const* words, const uint64_t* n_words, const vgc_group_hdr* const* hdrs,
                               uint32_t p, const vgc_group* groups, uint32_t n_groups, const void* plan,
                               float scale, int overwrite, float* dense_out, uint64_t n, void* stream, uint32_t tiles_per_wave) {
    if (!tiles_ok(tiles_per_wave)) return VGC_ERR_PARAM;
    if (!plan || !dense_out || (p && (!words || !n_words || !hdrs))) { set_error("vgc_unpack_add_batch: NULL pointer"); return VGC_ERR_NULL; }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    for (uint32_t w = 0; w < p; ++w) {
        if (!hdrs[w] || (!words[w] && n_words[w])) { set_error("vgc_unpack_add_batch: message %u has a NULL pointer", w); return VGC_ERR_NULL; }
        if (!aligned(words[w], 4) || !aligned(hdrs[w], 8)) { set_error("vgc_unpack_add_batch: message %u is misaligned", w); return VGC_ERR_ALIGN; }
    }
    if (!aligned(plan, 256) || !aligned(dense_out, 4)) { set_error("vgc_unpack_add_batch: misaligned pointer"); return VGC_ERR_ALIGN; }
    if (!std::isfinite(scale)) { set_error("vgc_unpack_add_batch: scale is not finite"); return VGC_ERR_PARAM; }
    if (p == 0 && !overwrite) return VGC_OK;
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    return launch_unpack_add_batch(plan_check(plan, gs), words, n_words, hdrs, p, pv.groups, pv.tiles, pv.runs, n_tiles, gs.n_runs, gs.whole_tiles, scale, overwrite, dense_out,
                                   tiles_per_wave, static_cast<hipStream_t>(stream));
}

int vgc_unpack_add_batch(const uint32_t* const* words, const uint64_t* n_words, const vgc_group_hdr* const* hdrs,
                         uint32_t p, const vgc_group* groups, uint32_t n_groups, const void* plan,
                         float scale, int overwrite, float* dense_out, uint64_t n, void* stream) {
    return vgc_tiles_unpack_add_batch(words, n_words, hdrs, p, groups, n_groups, plan, scale, overwrite, dense_out, n, stream, 0);
}

int vgc_tiles_unpack_apply(const uint32_t* const* words, const uint64_t* n_words, const vgc_group_hdr* const* hdrs,
                           uint32_t p, const vgc_group* groups, uint32_t n_groups, const void* plan, float scale,
                           const vgc_optimizer* opt, float* param, float* state1, float* state2, uint64_t n, void* stream,
                           uint32_t tiles_per_wave) {
    if (!tiles_ok(tiles_per_wave)) return VGC_ERR_PARAM;
    if (!plan || !opt || !param || !state1 || (p && (!words || !n_words || !hdrs))) { set_error("vgc_unpack_apply: NULL pointer"); return VGC_ERR_NULL; }
    if (opt->kind != VGC_OPT_MOMENTUM_SGD && opt->kind != VGC_OPT_ADAM) { set_error("vgc_unpack_apply: unknown optimizer %d", opt->kind); return VGC_ERR_PARAM; }
    if (opt->kind == VGC_OPT_ADAM && !state2) { set_error("vgc_unpack_apply: Adam needs state2"); return VGC_ERR_NULL; }
    if (p > VGC_MAX_UPDATE_MESSAGES) { set_error("vgc_unpack_apply: %u messages, at most %d", p, VGC_MAX_UPDATE_MESSAGES); return VGC_ERR_SIZE; }
    uint64_t n_tiles = 0;
    GroupStats gs;
    int rc = check_groups(groups, n_groups, n, &n_tiles, &gs);
    if (rc != VGC_OK) return rc;
    for (uint32_t w = 0; w < p; ++w) {
        if (!hdrs[w] || (!words[w] && n_words[w])) { set_error("vgc_unpack_apply: message %u has a NULL pointer", w); return VGC_ERR_NULL; }
        if (!aligned(words[w], 4) || !aligned(hdrs[w], 8)) { set_error("vgc_unpack_apply: message %u is misaligned", w); return VGC_ERR_ALIGN; }
    }
    if (!aligned(plan, 256) || !aligned(param, 4) || !aligned(state1, 4) || !aligned(state2, 4)) { set_error("vgc_unpack_apply: misaligned pointer"); return VGC_ERR_ALIGN; }
    if (!std::isfinite(scale) || !std::isfinite(opt->lr)) { set_error("vgc_unpack_apply: scale or lr is not finite"); return VGC_ERR_PARAM; }
    float mu = 0.f, b1 = 0.f, b2 = 0.f, omb1 = 0.f, omb2 = 0.f, bias1 = 1.f, bias2 = 1.f, eps = 0.f;
    if (opt->kind == VGC_OPT_MOMENTUM_SGD) {
        if (!(opt->momentum >= 0.0f) || !(opt->momentum < 1.0f)) { set_error("vgc_unpack_apply: need 0 <= momentum < 1 (got %g)", opt->momentum); return VGC_ERR_PARAM; }
        mu = opt->momentum;
    } else {
        if (!(opt->beta1 >= 0.0f) || !(opt->beta1 < 1.0f) || !(opt->beta2 >= 0.0f) || !(opt->beta2 < 1.0f) || !(opt->eps >= 0.0f) ||
            !std::isfinite(opt->eps) || opt->step < 1) {
            set_error("vgc_unpack_apply: need 0 <= beta1, beta2 < 1, eps >= 0, step >= 1");
            return VGC_ERR_PARAM;
        }
        b1 = opt->beta1; b2 = opt->beta2; eps = opt->eps;
        omb1 = (float)(1.0 - (double)b1);
        omb2 = (float)(1.0 - (double)b2);
        bias1 = (float)(1.0 - std::pow((double)b1, (double)opt->step));
        bias2 = (float)(1.0 - std::pow((double)b2, (double)opt->step));
    }
    const PlanView pv = plan_view(plan, n_tiles, n_groups);
    return launch_unpack_apply(plan_check(plan, gs), words, n_words, hdrs, p, pv.groups, pv.tiles, pv.runs, n_tiles, gs.n_runs, gs.whole_tiles, scale, opt->kind, opt->lr, mu, b1, b2,
                               omb1, omb2, bias1, bias2, eps, param, state1, state2, tiles_per_wave, static_cast<hipStream_t>(stream));
}

int vgc_unpack_apply(const uint32_t* const* words, const uint64_t* n_words, const vgc_group_hdr* const* hdrs,
                     uint32_t p, const vgc_group* groups, uint32_t n_groups, const void* plan, float scale,
                     const vgc_optimizer* opt, float* param, float* state1, float* state2, uint64_t n, void* stream) {
    return vgc_tiles_unpack_apply(words, n_words, hdrs, p, groups, n_groups, plan, scale, opt, param, state1, state2, n, stream, 0);
}

// ---- activations in 8 bits, layer norm, softmax loss ------------------------------------------------------------------------
static size_t element_bytes(int dtype) { return dtype == VGC_F32 ? 4 : 2; }

static int act8_check(const char* what, int dtype, const void* x, uint64_t R, uint32_t C, const void* codes, const void* exps) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("%s: unknown dtype %d", what, dtype); return VGC_ERR_DTYPE; }
    if (!x || !codes || !exps) { set_error("%s: the values, codes and exps are required", what); return VGC_ERR_NULL; }
    if (R == 0 || C == 0) { set_error("%s: zero dimension", what); return VGC_ERR_SIZE; }
    if (C > 0x7FFFFFFFu) { set_error("%s: rows of %u elements", what, C); return VGC_ERR_SIZE; }
    if (!aligned(x, element_bytes(dtype))) { set_error("%s: the values must be aligned to their elements", what); return VGC_ERR_ALIGN; }
    return VGC_OK;
}

int vgc_act8_encode(int dtype, const void* x, uint64_t R, uint32_t C, int8_t* codes, uint8_t* exps, void* stream) {
    const int rc = act8_check("vgc_act8_encode", dtype, x, R, C, codes, exps);
    return rc != VGC_OK ? rc : launch_act8_encode(dtype, x, R, C, codes, exps, static_cast<hipStream_t>(stream));
}

int vgc_act8_decode(int dtype, const int8_t* codes, const uint8_t* exps, uint64_t R, uint32_t C, void* out, void* stream) {
    const int rc = act8_check("vgc_act8_decode", dtype, out, R, C, codes, exps);
    return rc != VGC_OK ? rc : launch_act8_decode(dtype, codes, exps, R, C, out, static_cast<hipStream_t>(stream));
}

static int sqgrad_act8_shape(int kind, int dtype, uint32_t B, uint32_t P, uint32_t J, uint32_t C) {
    if (kind != VGC_FC && kind != VGC_CONV) { set_error("vgc_sqgrad_act8: unknown kind %d", kind); return VGC_ERR_DTYPE; }
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_sqgrad_act8: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (B == 0 || P == 0 || J == 0 || C == 0) { set_error("vgc_sqgrad_act8: zero dimension"); return VGC_ERR_SIZE; }
    if (kind == VGC_FC && P != 1) { set_error("vgc_sqgrad_act8: the FC form has P = 1"); return VGC_ERR_SIZE; }
    if (J > 65535u * 64u) { set_error("vgc_sqgrad_act8: J = %u exceeds the launch limit", J); return VGC_ERR_SIZE; }
    if (kind == VGC_FC && dtype == VGC_BF16 && !fc_planes_supported(B, J, C)) { set_error("vgc_sqgrad_act8: a row operand exceeds 2^31 bytes"); return VGC_ERR_SIZE; }
    return VGC_OK;
}

size_t vgc_sqgrad_act8_workspace_bytes(int kind, int dtype, uint32_t B, uint32_t P, uint32_t J, uint32_t C) {
    return sqgrad_act8_shape(kind, dtype, B, P, J, C) == VGC_OK ? sqgrad_act8_workspace_bytes(kind, dtype, B, P, J, C) : 0;
}

static int workspace_check(const char* what, const void* workspace, size_t workspace_bytes, size_t need) {
    if (!workspace && need) { set_error("%s: the workspace is required", what); return VGC_ERR_NULL; }
    if (workspace_bytes < need) { set_error("%s: workspace of %zu bytes, %zu needed", what, workspace_bytes, need); return VGC_ERR_SIZE; }
    if (!aligned(workspace, 16)) { set_error("%s: workspace must be 16-byte aligned", what); return VGC_ERR_ALIGN; }
    return VGC_OK;
}

int vgc_sqgrad_act8(int kind, int dtype, const int8_t* codes, const uint8_t* exps, const void* D, uint32_t B, uint32_t P, uint32_t J,
                    uint32_t C, float c, float* g_out, float* s_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!codes || !exps || !D || !s_out) { set_error("vgc_sqgrad_act8: codes, exps, D and s_out are required"); return VGC_ERR_NULL; }
    int rc = sqgrad_act8_shape(kind, dtype, B, P, J, C);
    if (rc != VGC_OK) return rc;
    if (!aligned(D, 16) || !aligned(s_out, 16) || (g_out && !aligned(g_out, 16))) {
        set_error("vgc_sqgrad_act8: D, s_out and g_out must be 16-byte aligned");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c)) { set_error("vgc_sqgrad_act8: c is not finite"); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_sqgrad_act8", workspace, workspace_bytes, sqgrad_act8_workspace_bytes(kind, dtype, B, P, J, C))) != VGC_OK) return rc;
    return launch_sqgrad_act8(kind, dtype, codes, exps, D, B, P, J, C, c, g_out, s_out, workspace, static_cast<hipStream_t>(stream));
}

int vgc_layer_norm(int dtype, const void* x, uint64_t R, uint32_t C, const float* gamma, const float* beta, float eps, void* y,
                   float* mean, float* rstd, int8_t* codes, uint8_t* exps, void* stream) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_layer_norm: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (!x || !gamma || !beta || !y || !mean || !rstd) { set_error("vgc_layer_norm: x, gamma, beta, y, mean and rstd are required"); return VGC_ERR_NULL; }
    if (!codes != !exps) { set_error("vgc_layer_norm: codes and exps go together"); return VGC_ERR_NULL; }
    if (R == 0 || C == 0) { set_error("vgc_layer_norm: zero dimension"); return VGC_ERR_SIZE; }
    if (R > 0x7FFFFFFFu || C > 0x7FFFFFFFu) { set_error("vgc_layer_norm: %llu rows of %u elements", (unsigned long long)R, C); return VGC_ERR_SIZE; }
    const size_t e = element_bytes(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) {
        set_error("vgc_layer_norm: pointers must be aligned to their elements");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(eps) || eps < 0.0f) { set_error("vgc_layer_norm: eps must be finite and not negative (got %g)", eps); return VGC_ERR_PARAM; }
    return launch_layer_norm(dtype, x, R, C, gamma, beta, eps, y, mean, rstd, codes, exps, static_cast<hipStream_t>(stream));
}

static int layer_norm_backward_shape(uint32_t B, uint32_t P, uint32_t C) {
    if (B == 0 || P == 0 || C == 0) { set_error("vgc_layer_norm_backward: zero dimension"); return VGC_ERR_SIZE; }
    if ((uint64_t)B * P > 0x7FFFFFFFull || C > 0x7FFFFFFFu) { set_error("vgc_layer_norm_backward: %u x %u rows of %u elements", B, P, C); return VGC_ERR_SIZE; }
    return VGC_OK;
}

size_t vgc_layer_norm_backward_workspace_bytes(uint32_t B, uint32_t P, uint32_t C) {
    return layer_norm_backward_shape(B, P, C) == VGC_OK ? layer_norm_backward_workspace_bytes(B, P, C) : 0;
}

int vgc_layer_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const int8_t* codes, const uint8_t* exps,
                            const float* rstd, const float* gamma, uint32_t B, uint32_t P, uint32_t C, float c, void* dx,
                            float* g_gamma, float* s_gamma, float* g_beta, float* s_beta, void* workspace, size_t workspace_bytes,
                            void* stream) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("vgc_layer_norm_backward: unknown dtype %d", dtype); return VGC_ERR_DTYPE; }
    if (!dy || !rstd || !gamma || !dx || !s_gamma || !s_beta) {
        set_error("vgc_layer_norm_backward: dy, rstd, gamma, dx, s_gamma and s_beta are required");
        return VGC_ERR_NULL;
    }
    if (!x != !mean || !codes != !exps || !x == !codes) {
        set_error("vgc_layer_norm_backward: the rows come as x and mean or as codes and exps");
        return VGC_ERR_NULL;
    }
    int rc = layer_norm_backward_shape(B, P, C);
    if (rc != VGC_OK) return rc;
    const size_t e = element_bytes(dtype);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(gamma, 4) ||
        !aligned(g_gamma, 4) || !aligned(s_gamma, 4) || !aligned(g_beta, 4) || !aligned(s_beta, 4)) {
        set_error("vgc_layer_norm_backward: pointers must be aligned to their elements");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c)) { set_error("vgc_layer_norm_backward: c is not finite"); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_layer_norm_backward", workspace, workspace_bytes, layer_norm_backward_workspace_bytes(B, P, C))) != VGC_OK) return rc;
    return launch_layer_norm_backward(dtype, dy, x, mean, codes, exps, rstd, gamma, B, P, C, c, dx, g_gamma, s_gamma, g_beta, s_beta, workspace,
                                      static_cast<hipStream_t>(stream));
}

static int softmax_loss_shape(const char* what, int dtype, uint32_t B, uint32_t P, uint32_t H, uint32_t V) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("%s: unknown dtype %d", what, dtype); return VGC_ERR_DTYPE; }
    if (B == 0 || P == 0 || H == 0 || V == 0) { set_error("%s: zero dimension", what); return VGC_ERR_SIZE; }
    // (padded to whole steps and cut into six pieces, a tile's 256 rows of any operand stay below 2^32 bytes)
    if ((uint64_t)B * ((P + 31ull) / 32u * 32u) > (1u << 20) && P > 1) { set_error("%s: %u x %u positions exceed 2^20", what, B, P); return VGC_ERR_SIZE; }
    if ((uint64_t)B * P > (1u << 20) || H > (1u << 20)) { set_error("%s: %u x %u rows of %u elements exceed 2^20", what, B, P, H); return VGC_ERR_SIZE; }
    if (V > (1u << 24)) { set_error("%s: %u classes exceed 2^24", what, V); return VGC_ERR_SIZE; }
    return VGC_OK;
}

size_t vgc_softmax_loss_workspace_bytes(int dtype, uint32_t N, uint32_t H, uint32_t V) {
    return softmax_loss_shape("vgc_softmax_loss", dtype, N, 1, H, V) == VGC_OK ? softmax_loss_workspace_bytes(dtype, N, H, V) : 0;
}

int vgc_softmax_loss(int dtype, const void* X, const void* W, const int64_t* target, uint32_t N, uint32_t H, uint32_t V, float* loss,
                     float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !W || !target || !loss || !lse) { set_error("vgc_softmax_loss: X, W, target, loss and lse are required"); return VGC_ERR_NULL; }
    int rc = softmax_loss_shape("vgc_softmax_loss", dtype, N, 1, H, V);
    if (rc != VGC_OK) return rc;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(target, 8) || !aligned(loss, 4) || !aligned(lse, 4)) {
        set_error("vgc_softmax_loss: X and W must be 16-byte aligned, the others to their elements");
        return VGC_ERR_ALIGN;
    }
    if ((rc = workspace_check("vgc_softmax_loss", workspace, workspace_bytes, softmax_loss_workspace_bytes(dtype, N, H, V))) != VGC_OK) return rc;
    return launch_softmax_loss(dtype, X, W, target, N, H, V, loss, lse, workspace, static_cast<hipStream_t>(stream));
}

size_t vgc_softmax_loss_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t H, uint32_t V) {
    return softmax_loss_shape("vgc_softmax_loss_backward", dtype, B, P, H, V) == VGC_OK ? softmax_loss_backward_workspace_bytes(dtype, B, P, H, V) : 0;
}

int vgc_softmax_loss_backward(int dtype, const void* X, const void* W, const int64_t* target, const float* lse, const float* weight,
                              uint32_t B, uint32_t P, uint32_t H, uint32_t V, float c, void* dX, float* g_out, float* s_out,
                              void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !W || !target || !lse) { set_error("vgc_softmax_loss_backward: X, W, target and lse are required"); return VGC_ERR_NULL; }
    if ((!dX && !s_out) || (g_out && !s_out)) { set_error("vgc_softmax_loss_backward: dX or s_out is required, and s_out with g_out"); return VGC_ERR_NULL; }
    int rc = softmax_loss_shape("vgc_softmax_loss_backward", dtype, B, P, H, V);
    if (rc != VGC_OK) return rc;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(dX, 16) || !aligned(g_out, 16) || !aligned(s_out, 16) || !aligned(target, 8) ||
        !aligned(lse, 4) || !aligned(weight, 4)) {
        set_error("vgc_softmax_loss_backward: X, W, dX, g_out and s_out must be 16-byte aligned, the others to their elements");
        return VGC_ERR_ALIGN;
    }
    if (!std::isfinite(c)) { set_error("vgc_softmax_loss_backward: c is not finite"); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_softmax_loss_backward", workspace, workspace_bytes, softmax_loss_backward_workspace_bytes(dtype, B, P, H, V))) != VGC_OK) return rc;
    return launch_softmax_loss_backward(dtype, X, W, target, lse, weight, B, P, H, V, c, dX, g_out, s_out, workspace, static_cast<hipStream_t>(stream));
}

// ---- linear layer, dropout, group norm ----------------------------------------------------------------------------------------
static int type_check(const char* what, int dtype) {
    if (dtype != VGC_F32 && dtype != VGC_BF16) { set_error("%s: unknown dtype %d", what, dtype); return VGC_ERR_DTYPE; }
    return VGC_OK;
}
static int act_check(const char* what, int act) {
    if (act < VGC_ACT_NONE || act > VGC_ACT_SILU) { set_error("%s: unknown activation %d", what, act); return VGC_ERR_PARAM; }
    return VGC_OK;
}
static int dropout_check(const char* what, float p, const uint64_t* rng) {
    if (!(p >= 0.0f && p <= 1.0f)) { set_error("%s: p must be in [0, 1] (got %g)", what, p); return VGC_ERR_PARAM; }
    if (dropout_of(p, rng).t != 0u && !rng) { set_error("%s: rng is required where elements are dropped", what); return VGC_ERR_NULL; }
    if (!aligned(rng, 8)) { set_error("%s: rng must be aligned to its elements", what); return VGC_ERR_ALIGN; }
    return VGC_OK;
}

int vgc_dropout(int dtype, const void* x, const void* residual, uint64_t R, uint32_t C, float p, const uint64_t* rng, void* y, void* stream) {
    int rc = type_check("vgc_dropout", dtype);
    if (rc != VGC_OK) return rc;
    if (!x || !y) { set_error("vgc_dropout: x and y are required"); return VGC_ERR_NULL; }
    if (R == 0 || C == 0) { set_error("vgc_dropout: zero dimension"); return VGC_ERR_SIZE; }
    if (R > 0x7FFFFFFFu || C > 0x7FFFFFFFu) { set_error("vgc_dropout: %llu rows of %u elements", (unsigned long long)R, C); return VGC_ERR_SIZE; }
    const size_t e = element_bytes(dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(y, e)) { set_error("vgc_dropout: pointers must be aligned to their elements"); return VGC_ERR_ALIGN; }
    if ((rc = dropout_check("vgc_dropout", p, rng)) != VGC_OK) return rc;
    return launch_dropout(dtype, x, residual, (uint32_t)R, C, dropout_of(p, rng), y, static_cast<hipStream_t>(stream));
}

static int linear_shape(const char* what, int dtype, uint32_t B, uint32_t P, uint32_t K, uint32_t C) {
    const int rc = type_check(what, dtype);
    if (rc != VGC_OK) return rc;
    if (B == 0 || P == 0 || K == 0 || C == 0) { set_error("%s: zero dimension", what); return VGC_ERR_SIZE; }
    const uint64_t N = (uint64_t)B * P;
    if (N > (1u << 20) || K > (1u << 20) || C > (1u << 20)) { set_error("%s: %llu rows, %u to %u columns exceed 2^20", what, (unsigned long long)N, K, C); return VGC_ERR_SIZE; }
    if ((uint64_t)K * C > (1u << 30)) { set_error("%s: a weight of %u x %u exceeds 2^30", what, K, C); return VGC_ERR_SIZE; }
    if (N * K > (1ull << 34) || N * C > (1ull << 34)) { set_error("%s: %llu rows of %u and %u columns exceed 2^34", what, (unsigned long long)N, K, C); return VGC_ERR_SIZE; }
    return VGC_OK;
}

size_t vgc_linear_workspace_bytes(int dtype, uint32_t N, uint32_t K, uint32_t C) {
    return linear_shape("vgc_linear", dtype, N, 1, K, C) == VGC_OK ? linear_workspace_bytes(dtype, N, K, C) : 0;
}

int vgc_linear(int dtype, const void* X, const void* W, const float* bias, int act, float p, const uint64_t* rng, const void* residual, uint32_t N,
               uint32_t K, uint32_t C, void* z, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !W || !y) { set_error("vgc_linear: X, W and y are required"); return VGC_ERR_NULL; }
    int rc = linear_shape("vgc_linear", dtype, N, 1, K, C);
    if (rc != VGC_OK) return rc;
    const size_t e = element_bytes(dtype);
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(bias, 4) || !aligned(residual, e) || !aligned(z, e) || !aligned(y, e)) {
        set_error("vgc_linear: X and W must be 16-byte aligned, the others to their elements");
        return VGC_ERR_ALIGN;
    }
    if ((rc = act_check("vgc_linear", act)) != VGC_OK || (rc = dropout_check("vgc_linear", p, rng)) != VGC_OK) return rc;
    if ((rc = workspace_check("vgc_linear", workspace, workspace_bytes, linear_workspace_bytes(dtype, N, K, C))) != VGC_OK) return rc;
    LinearCall L = {};
    L.dtype = dtype; L.act = act; L.X = X; L.W = W; L.residual = residual; L.bias = bias; L.p = p; L.rng = rng;
    L.B = N; L.P = 1; L.K = K; L.C = C; L.z = z; L.y = y;
    return launch_linear(L, workspace, static_cast<hipStream_t>(stream));
}

size_t vgc_linear_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t K, uint32_t C) {
    return linear_shape("vgc_linear_backward", dtype, B, P, K, C) == VGC_OK ? linear_backward_workspace_bytes(dtype, B, P, K, C) : 0;
}

int vgc_linear_backward(int dtype, const void* dy, const void* z, const void* W, int act, float p, const uint64_t* rng, const void* add, uint32_t B,
                        uint32_t P, uint32_t K, uint32_t C, float c, void* dz, void* dX, float* g_bias, float* s_bias, void* workspace,
                        size_t workspace_bytes, void* stream) {
    if (!dy || !dz || (dX && !W)) { set_error("vgc_linear_backward: dy and dz are required, and W for dX"); return VGC_ERR_NULL; }
    if ((g_bias && !s_bias) || (add && !dX)) { set_error("vgc_linear_backward: g_bias goes with s_bias, and add with dX"); return VGC_ERR_NULL; }
    int rc = linear_shape("vgc_linear_backward", dtype, B, P, K, C);
    if (rc != VGC_OK) return rc;
    if ((rc = act_check("vgc_linear_backward", act)) != VGC_OK) return rc;
    if (act != VGC_ACT_NONE && !z) { set_error("vgc_linear_backward: z is required with an activation"); return VGC_ERR_NULL; }
    const size_t e = element_bytes(dtype);
    if (!aligned(W, 16) || !aligned(dz, 16) || !aligned(dy, e) || !aligned(z, e) || !aligned(add, e) || !aligned(dX, e) || !aligned(g_bias, 4) || !aligned(s_bias, 4)) {
        set_error("vgc_linear_backward: W and dz must be 16-byte aligned, the others to their elements");
        return VGC_ERR_ALIGN;
    }
    if ((rc = dropout_check("vgc_linear_backward", p, rng)) != VGC_OK) return rc;
    if (!std::isfinite(c)) { set_error("vgc_linear_backward: c is not finite"); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_linear_backward", workspace, workspace_bytes, linear_backward_workspace_bytes(dtype, B, P, K, C))) != VGC_OK) return rc;
    LinearCall L = {};
    L.dtype = dtype; L.act = act; L.W = W; L.residual = add; L.dy = dy; L.z_in = z; L.p = p; L.c = c; L.rng = rng;
    L.B = B; L.P = P; L.K = K; L.C = C; L.dz = dz; L.dX = dX; L.g_bias = g_bias; L.s_bias = s_bias;
    return launch_linear_backward(L, workspace, static_cast<hipStream_t>(stream));
}

static int group_norm_shape(const char* what, int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    const int rc = type_check(what, dtype);
    if (rc != VGC_OK) return rc;
    if (B == 0 || P == 0 || C == 0 || G == 0) { set_error("%s: zero dimension", what); return VGC_ERR_SIZE; }
    if ((uint64_t)B * P > 0x7FFFFFFFull || C > (1u << 20)) { set_error("%s: %u x %u positions of %u channels", what, B, P, C); return VGC_ERR_SIZE; }
    if (C % G != 0) { set_error("%s: %u channels are not %u groups of one size", what, C, G); return VGC_ERR_SIZE; }
    return VGC_OK;
}

size_t vgc_group_norm_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    return group_norm_shape("vgc_group_norm", dtype, B, P, C, G) == VGC_OK ? group_norm_workspace_bytes(dtype, B, P, C, G) : 0;
}

int vgc_group_norm(int dtype, const void* x, uint32_t B, uint32_t P, uint32_t C, uint32_t G, const float* gamma, const float* beta, float eps, int act,
                   void* y, float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !gamma || !beta || !y || !mean || !rstd) { set_error("vgc_group_norm: x, gamma, beta, y, mean and rstd are required"); return VGC_ERR_NULL; }
    int rc = group_norm_shape("vgc_group_norm", dtype, B, P, C, G);
    if (rc != VGC_OK) return rc;
    const size_t e = element_bytes(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) {
        set_error("vgc_group_norm: pointers must be aligned to their elements");
        return VGC_ERR_ALIGN;
    }
    if ((rc = act_check("vgc_group_norm", act)) != VGC_OK) return rc;
    if (!std::isfinite(eps) || eps < 0.0f) { set_error("vgc_group_norm: eps must be finite and not negative (got %g)", eps); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_group_norm", workspace, workspace_bytes, group_norm_workspace_bytes(dtype, B, P, C, G))) != VGC_OK) return rc;
    return launch_group_norm(dtype, x, B, P, C, G, gamma, beta, eps, act, y, mean, rstd, workspace, static_cast<hipStream_t>(stream));
}

size_t vgc_group_norm_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    return group_norm_shape("vgc_group_norm_backward", dtype, B, P, C, G) == VGC_OK ? group_norm_backward_workspace_bytes(dtype, B, P, C, G) : 0;
}

int vgc_group_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma, const float* beta, int act,
                            uint32_t B, uint32_t P, uint32_t C, uint32_t G, float c, void* dx, float* g_gamma, float* s_gamma, float* g_beta,
                            float* s_beta, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy || !x || !mean || !rstd || !gamma || !beta || !dx || !s_gamma || !s_beta) {
        set_error("vgc_group_norm_backward: dy, x, mean, rstd, gamma, beta, dx, s_gamma and s_beta are required");
        return VGC_ERR_NULL;
    }
    int rc = group_norm_shape("vgc_group_norm_backward", dtype, B, P, C, G);
    if (rc != VGC_OK) return rc;
    const size_t e = element_bytes(dtype);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(gamma, 4) || !aligned(beta, 4) ||
        !aligned(g_gamma, 4) || !aligned(s_gamma, 4) || !aligned(g_beta, 4) || !aligned(s_beta, 4)) {
        set_error("vgc_group_norm_backward: pointers must be aligned to their elements");
        return VGC_ERR_ALIGN;
    }
    if ((rc = act_check("vgc_group_norm_backward", act)) != VGC_OK) return rc;
    if (!std::isfinite(c)) { set_error("vgc_group_norm_backward: c is not finite"); return VGC_ERR_PARAM; }
    if ((rc = workspace_check("vgc_group_norm_backward", workspace, workspace_bytes, group_norm_backward_workspace_bytes(dtype, B, P, C, G))) != VGC_OK) return rc;
    return launch_group_norm_backward(dtype, dy, x, mean, rstd, gamma, beta, act, B, P, C, G, c, dx, g_gamma, s_gamma, g_beta, s_beta, workspace,
                                      static_cast<hipStream_t>(stream));
}

// Not in vgc.h: which of its forms a call takes, for tests that have to reach them all.
int vgc_form_group_norm(int dtype, int backward, uint32_t B, uint32_t P, uint32_t C, uint32_t G, uint32_t* form) {
    const int rc = group_norm_shape("vgc_form_group_norm", dtype, B, P, C, G);
    if (rc == VGC_OK) group_norm_form(dtype, backward != 0, B, P, C, G, form);
    return rc;
}

int vgc_form_linear(int dtype, int backward, uint32_t B, uint32_t P, uint32_t K, uint32_t C, uint32_t* form) {
    const int rc = linear_shape("vgc_form_linear", dtype, B, P, K, C);
    if (rc == VGC_OK) linear_form(dtype, backward != 0, B, P, K, C, form);
    return rc;
}

}  // extern "C"
