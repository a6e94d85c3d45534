// Host-only harness around the encoder and decoder of 8-bit records.
#include <cstring>
#include <new>

#include "../../paper_2607_08786_amd/csrc/usp_internal.h"

extern "C" {

// Encodes, copies the records (at most stream_cap bytes) and the offsets, decodes back. 0 on success.
int usp_test_q(const int8_t *W, int64_t ldw, const uint8_t *mask, int64_t ldm, int64_t M, int64_t K, int8_t *W_out,
               uint8_t *mask_out, int64_t *nnz, uint8_t *stream_out, int64_t stream_cap, uint32_t *off_out) {
    usp::HostEncoding enc;
    try {
        usp::encode_host_q(W, ldw, mask, ldm, M, K, enc);
    } catch (const std::bad_alloc &) {
        return 1;
    }
    if ((int64_t)enc.stream.size() > stream_cap) return 3;
    *nnz = enc.nnz;
    std::memcpy(stream_out, enc.stream.data(), enc.stream.size());
    std::memcpy(off_out, enc.off.data(), enc.off.size() * sizeof(uint32_t));
    return usp::decode_host_q(enc, W_out, mask_out) ? 0 : 2;
}
}
