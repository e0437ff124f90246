// C entry points of the attention with decaying states: argument checks, kernel choice, launches.
#include "ccv3d_tokens_decay_tile.cuh"
#include "ccv3d_tokens_host.cuh"

using namespace ccv3d;

namespace {

struct DecayPlan {
    Device dev;
    bool step;
    int columns;                 // value columns of a chunk block
    int seg;                     // tokens of a segment, 0: not cut
    int64_t items, fade_at;
    uint64_t bytes;
};

ccv3d_status check_decay(const ccv3d_decay_memory* m, const ccv3d_stream_batch* b, int qk_heads, int dtype) {
    if (!m || !m->states || m->slots < 1 || m->heads < 1 || !b || b->batch < 0 || b->tokens < 0 || b->max_new < 0) return CCV3D_ERR_INVALID_ARG;
    if (!dtype_ok(dtype) || qk_heads < 1 || m->heads % qk_heads) return CCV3D_ERR_INVALID_ARG;
    if (m->key_dim != 64 && m->key_dim != 128) return CCV3D_ERR_UNSUPPORTED;
    if (m->value_dim < 64 || m->value_dim % 64 || m->value_dim > 512 || m->heads > 4096) return CCV3D_ERR_UNSUPPORTED;
    if (misaligned(m->states, 16)) return CCV3D_ERR_ALIGNMENT;
    if (b->batch == 0) return b->tokens == 0 ? CCV3D_OK : CCV3D_ERR_INVALID_ARG;
    if (b->batch > 65536 || b->tokens > (1 << 30)) return CCV3D_ERR_UNSUPPORTED;
    if (!b->new_start || !b->slot) return CCV3D_ERR_INVALID_ARG;
    if (misaligned(b->new_start, 4) || misaligned(b->slot, 4) || misaligned(b->fresh, 4)) return CCV3D_ERR_ALIGNMENT;
    return CCV3D_OK;
}

ccv3d_status plan_decay(const ccv3d_decay_memory* m, const ccv3d_stream_batch* b, int dtype, DecayPlan* q) {
    const ccv3d_status s = current_device(&q->dev);
    if (s != CCV3D_OK) return s;
    // Up to which number of new tokens a state goes token by token.  us, 64 sequences of n tokens, 32 heads of 128 (16 of 64), step kernel /
    // chunks, BF16: 9 tokens 87 / 155 (17 / 56), 16 119 / 156 (21 / 56), 32 204 / 159 (37 / 56), 64 377 / 164 (66 / 58);
    // F32: 16 122 / 271 (21 / 58), 64 378 / 411 (72 / 84), 128 721 / 726 (136 / 170)
    q->step = b->max_new <= (dtype == CCV3D_F32 ? 128 : 24);
    q->columns = dtype == CCV3D_BF16 || m->value_dim % 128 == 0 ? 128 : 64;
    q->seg = 0;
    q->items = q->fade_at = 0;
    q->bytes = 0;
    if (q->step) return CCV3D_OK;
    // Where the sequences do not fill the machine they are cut so that one turn of blocks does: a block's start and end cost as much as some
    // chunks.  Where one may be far longer than the others, segments are four times as long as their mean, so that not much else is cut
    // (max_new is a bound, and may say so of sequences that are all alike).
    const int64_t wide = (int64_t)m->heads * ((m->value_dim + q->columns - 1) / q->columns), fit = q->dev.sm_count, B = b->batch;
    const int64_t longest = b->max_new < b->tokens ? b->max_new : b->tokens, mean = b->tokens / B + 64;
    int64_t per;
    if (wide * B < fit) {
        const int64_t items = fit / wide > B ? fit / wide : B, chunks = (b->tokens + DECAY_CHUNK - 1) / DECAY_CHUNK;
        per = (chunks + items - 1) / items;
    } else {
        if (longest <= 8 * mean) return CCV3D_OK;
        per = 4 * mean / DECAY_CHUNK;
    }
    if (per < 4) per = 4;
    if (per * DECAY_CHUNK >= longest) return CCV3D_OK;
    // Items are segments of sequences of more than one: no more than tokens / seg, and one more for each such sequence.
    q->seg = (int)(per * DECAY_CHUNK);
    const int64_t cut = b->tokens / (q->seg + 1);
    q->items = b->tokens / q->seg + (cut < B ? cut : B);
    q->fade_at = (q->items * m->heads * m->key_dim * m->value_dim * 4 + 255) / 256 * 256;
    q->bytes = (uint64_t)(q->fade_at + (q->items * m->heads * 4 + 255) / 256 * 256);
    return CCV3D_OK;
}

// A pass over the chunks of sequences or items: BF16 on tcgen05, F32 by mma.sync, with eight or four warps to 128 or 64 value columns.
template <typename T, int DK, int MODE>
ccv3d_status launch_chunks(const DecayParams& p, const DecayPlan& q, int64_t items, cudaStream_t st) {
    const dim3 grid((unsigned)items, p.m.heads * ((p.m.value_dim + q.columns - 1) / q.columns));
    const auto launch = [&](auto* kernel, int threads, int bytes, std::atomic<uint64_t>& done) {
        if (!allow_smem(kernel, bytes, q.dev.index, done)) { cudaGetLastError(); return CCV3D_ERR_CUDA; }
        kernel<<<grid, threads, bytes, st>>>(p);
        return launched();
    };
    static std::atomic<uint64_t> done[2];
    if constexpr (sizeof(T) == 2) return launch(decay_tile_kernel<DK, MODE>, DECAY_TILE_THREADS, DecayTileShape<DK>::SHARED_AT + sizeof(DecayTileShared), done[0]);
    else if (q.columns == 128) return launch(decay_chunk_kernel<DK, 8, MODE>, 256, DecayShape<DK, 8>::BYTES, done[0]);
    else return launch(decay_chunk_kernel<DK, 4, MODE>, 128, DecayShape<DK, 4>::BYTES, done[1]);
}

template <typename T, int DK>
ccv3d_status launch_prompt(const DecayParams& p, const DecayPlan& q, cudaStream_t st) {
    if (!q.seg) return launch_chunks<T, DK, DECAY_OUTPUTS>(p, q, p.bt.batch, st);
    ccv3d_status s = launch_chunks<T, DK, DECAY_STATES>(p, q, q.items, st);
    if (s != CCV3D_OK) return s;
    const int64_t size = (int64_t)DK * p.m.value_dim;
    decay_scan_kernel<<<dim3(p.bt.batch, (unsigned)((size + 1023) / 1024), p.m.heads), DECAY_SCAN_THREADS, 0, st>>>(p);
    if ((s = launched()) != CCV3D_OK) return s;
    return launch_chunks<T, DK, DECAY_OUTPUTS>(p, q, q.items + p.bt.batch, st);
}

template <typename T, int DK>
ccv3d_status launch_decay(const DecayParams& p, const DecayPlan& q, cudaStream_t st) {
    if (q.step) {
        const int64_t blocks = (int64_t)p.bt.batch * p.m.heads * (p.m.value_dim / 64);
        if (blocks > 0x7FFFFFFF) return CCV3D_ERR_UNSUPPORTED;
        decay_step_kernel<T, DK><<<(unsigned)blocks, DECAY_STEP_THREADS, 0, st>>>(p);
        return launched();
    }
    return launch_prompt<T, DK>(p, q, st);
}

}  // namespace

extern "C" {

ccv3d_status ccv3d_decay_attend_workspace(const ccv3d_decay_memory* memory, const ccv3d_stream_batch* batch, int32_t qk_heads,
                                          int32_t dtype, uint64_t* bytes_host) {
    if (!bytes_host) return CCV3D_ERR_INVALID_ARG;
    ccv3d_status s = check_decay(memory, batch, qk_heads, dtype);
    if (s != CCV3D_OK) return s;
    *bytes_host = 0;
    if (batch->batch == 0) return s;
    DecayPlan q;
    if ((s = plan_decay(memory, batch, dtype, &q)) == CCV3D_OK) *bytes_host = q.bytes;
    return s;
}

ccv3d_status ccv3d_decay_attend(const ccv3d_decay_memory* memory, const ccv3d_stream_batch* batch, const ccv3d_heads* q,
                                const ccv3d_heads* k, const ccv3d_heads* v, const float* log_decay, int64_t decay_token_stride,
                                int64_t decay_head_stride, const ccv3d_heads* out, int32_t qk_heads, int32_t dtype, float scale,
                                void* ws, uint64_t ws_bytes, uint32_t* status, void* stream) {
    ccv3d_status s = check_decay(memory, batch, qk_heads, dtype);
    if (s != CCV3D_OK) return s;
    const int64_t tokens = batch->tokens;
    if (tokens == 0 || batch->max_new == 0) return CCV3D_OK;
    const int H = memory->heads, DK = memory->key_dim, DV = memory->value_dim;
    if (!log_decay || decay_token_stride < 0 || decay_head_stride < 0) return CCV3D_ERR_INVALID_ARG;
    if ((s = check_heads(q, qk_heads, DK, dtype)) != CCV3D_OK || (s = check_heads(k, qk_heads, DK, dtype)) != CCV3D_OK ||
        (s = check_heads(v, H, DV, dtype)) != CCV3D_OK || (s = check_heads(out, H, DV, dtype, tokens)) != CCV3D_OK)
        return s;
    if (misaligned(log_decay, 4) || misaligned(status, 4)) return CCV3D_ERR_ALIGNMENT;
    DecayPlan pl;
    if ((s = plan_decay(memory, batch, dtype, &pl)) != CCV3D_OK) return s;
    if ((s = check_ws(ws, ws_bytes, pl.bytes)) != CCV3D_OK) return s;
    const Span so = span_of(*out, tokens, H, DV, dtype), ss = span_of(memory->states, (int64_t)memory->slots * H * DK * DV * 4), sw = span_of(ws, (int64_t)pl.bytes);
    const Span in[] = {span_of(*q, tokens, qk_heads, DK, dtype), span_of(*k, tokens, qk_heads, DK, dtype), span_of(*v, tokens, H, DV, dtype),
                       span_of(log_decay, ((tokens - 1) * decay_token_stride + (H - 1) * decay_head_stride + 1) * 4),
                       span_of(batch->new_start, (batch->batch + 1LL) * 4), span_of(batch->slot, batch->batch * 4LL),
                       span_of(batch->fresh, batch->fresh ? batch->batch * 4LL : 0)};
    for (const Span& t : in)
        if (t.a != t.b && (meet(t, so) || meet(t, ss) || (pl.bytes && meet(t, sw)))) return CCV3D_ERR_ALIAS;
    if (meet(so, ss) || (pl.bytes && (meet(sw, so) || meet(sw, ss)))) return CCV3D_ERR_ALIAS;
    DecayParams p = {};
    p.m = *memory;
    p.bt = *batch;
    p.q = *q;
    p.k = *k;
    p.v = *v;
    p.o = *out;
    p.decay = log_decay;
    p.d_token = decay_token_stride;
    p.d_head = decay_head_stride;
    p.group = H / qk_heads;
    p.scale = scale;
    p.status = status;
    p.wait_clk = pl.dev.wait_clk;
    p.seg = pl.seg;
    p.items = (int)pl.items;
    p.part = (float*)ws;
    p.fade = (float*)((char*)ws + pl.fade_at);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == CCV3D_BF16) return DK == 64 ? launch_decay<__nv_bfloat16, 64>(p, pl, st) : launch_decay<__nv_bfloat16, 128>(p, pl, st);
    return DK == 64 ? launch_decay<float, 64>(p, pl, st) : launch_decay<float, 128>(p, pl, st);
}

}  // extern "C"
