// Host side of the layer's calls: what their argument checks and workspaces share.
#pragma once
#include "layer.hpp"

namespace last {
void note_hip_error(hipError_t e);
int option(int o);
}

namespace {

using namespace last;

constexpr long long kMaxRows = 1ll << 30;
constexpr long long kMaxColumns = 1ll << 20;
constexpr long long kMaxPitchBytes = 4ll << 20;      // 256 rows of a tile stay within 32-bit offsets
constexpr size_t kAlign = 256;
constexpr long long kMaxThreads = 1ll << 31;         // of a launch, which takes fewer than 2^32: what has more to do goes out in pieces

size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

last_status_t hip_done()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LAST_OK;
    note_hip_error(e);
    return LAST_ERR_HIP;
}

bool plain(int t) { return t == LAST_F32 || t == LAST_BF16 || t == LAST_F16; }
bool half_width(int t) { return t == LAST_BF16 || t == LAST_F16; }
bool eight(int t) { return t == LAST_I8 || t == LAST_E4M3; }
int size_of(int t) { return t == LAST_F32 ? 4 : half_width(t) ? 2 : 1; }

last_status_t check_frames(const last_frames_t* f, long long* rows)
{
    if (!f) return LAST_ERR_NULL;
    if (f->B < 1 || f->T < 0 || (long long)f->B * f->T > kMaxRows) return LAST_ERR_SHAPE;
    *rows = (long long)f->B * f->T;
    return LAST_OK;
}

last_status_t check_matrix(const last_matrix_t* m, long long columns, bool types)
{
    if (!m || !m->data) return LAST_ERR_NULL;
    if (!types) return LAST_ERR_UNSUPPORTED;
    if (m->pitch < columns || m->pitch > kMaxPitchBytes / size_of(m->type)) return LAST_ERR_SHAPE;
    if ((uintptr_t)m->data % size_of(m->type) != 0) return LAST_ERR_SHAPE;
    if (eight(m->type)) {
        if (!m->scales) return LAST_ERR_NULL;
        if (m->scale_pitch < (columns + kBlock - 1) / kBlock || m->scale_pitch > kMaxPitchBytes) return LAST_ERR_SHAPE;
    }
    return LAST_OK;
}

#define LAST_TRY(call)                                  \
    do {                                                \
        const last_status_t rc_ = (call);               \
        if (rc_ != LAST_OK) return rc_;                 \
    } while (0)

Frames frames_of(const last_frames_t* f) { return Frames{f->lengths, f->T, divisor_of((unsigned)f->T)}; }

Eight eight_of(const last_matrix_t* m)
{
    Eight e{};
    if (!m) return e;
    e.q = (uint8_t*)m->data;
    e.scales = m->scales;
    e.pitch = m->pitch;
    e.scale_pitch = m->scale_pitch;
    e.e4m3 = m->type == LAST_E4M3;
    return e;
}

struct Carver {
    char* base;
    size_t have, used = 0;
    explicit Carver(void* p, size_t n = 0) : base((char*)p), have(n) {}
    // a plan that went by another setting of an option than the size that was checked (set in between, by another thread)
    bool over() const { return base && used > have; }
    char* take(size_t bytes)
    {
        char* p = base ? base + used : nullptr;
        used += align_up(bytes);
        return p;
    }
};

// need 0: sizes that no plan takes (the rest is checked by then)
last_status_t check_ws(void* ws, size_t have, size_t need)
{
    if (need == 0) return LAST_ERR_SHAPE;
    if (!ws || ((uintptr_t)ws % kAlign) != 0 || have < need) return LAST_ERR_WORKSPACE;
    return LAST_OK;
}

}  // namespace
