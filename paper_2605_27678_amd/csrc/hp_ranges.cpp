// Which packed image tokens each position of a sequence sees (host only).
#include <cstdint>

#include "hp_operators.h"

namespace {

// Fills in one sample's positions: images [begin, end) of the map, whose tokens begin at packed row `base`.
void sample_ranges(const hp_token_map_t &m, int32_t begin, int32_t end, int64_t base, int32_t rule, int32_t *ranges) {
    int64_t all = base;
    for (int32_t k = begin; k < end; ++k) all += m.img_len[k];
    if (rule == HP_SEE_SAMPLE) {
        for (int32_t p = 0; p < m.seq; ++p) {
            ranges[2 * (int64_t)p] = (int32_t)base;
            ranges[2 * (int64_t)p + 1] = (int32_t)all;
        }
        return;
    }
    int64_t first = base, seen = base;                // of the latest image's tokens, and behind them
    int32_t k = begin;
    for (int32_t p = 0; p < m.seq; ++p) {
        while (k < end && (int64_t)m.img_start[k] + m.img_len[k] <= p) {
            first = seen;
            seen += m.img_len[k++];
        }
        ranges[2 * (int64_t)p] = (int32_t)(rule == HP_SEE_LATEST ? first : base);
        ranges[2 * (int64_t)p + 1] = (int32_t)seen;
    }
}

}  // namespace

extern "C" int hp_image_ranges(const hp_token_map_t *m, int32_t rule, int32_t *ranges) {
    if (!m || !ranges || m->batch < 1 || m->seq < 1 || m->n_images < 0) return HP_EINVAL;
    if (m->n_images > 0 && (!m->img_sample || !m->img_start || !m->img_len)) return HP_EINVAL;
    if (rule < HP_SEE_SAMPLE || rule > HP_SEE_LATEST) return HP_EINVAL;
    int64_t tokens = 0;
    for (int32_t k = 0; k < m->n_images; ++k) {
        const int32_t b = m->img_sample[k];
        const int64_t s = m->img_start[k], n = m->img_len[k];
        if (b < 0 || b >= m->batch || (k && b < m->img_sample[k - 1])) return HP_EMAP;
        if (s < 0 || n < 1 || s + n > m->seq) return HP_EMAP;
        if (rule != HP_SEE_SAMPLE && k && b == m->img_sample[k - 1] && s < (int64_t)m->img_start[k - 1] + m->img_len[k - 1]) return HP_EMAP;
        tokens += n;
    }
    if (tokens > INT32_MAX) return HP_ELAYOUT;
    int32_t k = 0;
    int64_t base = 0;
    for (int32_t b = 0; b < m->batch; ++b) {
        int32_t end = k;
        int64_t next = base;
        while (end < m->n_images && m->img_sample[end] == b) next += m->img_len[end++];
        sample_ranges(*m, k, end, base, rule, ranges + 2 * (int64_t)b * m->seq);
        k = end;
        base = next;
    }
    return HP_OK;
}
