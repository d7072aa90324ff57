"""Torch plumbing around the C ABI: device allocations (weights, paged KV cache, block table,
workspace) and tensor-level wrappers of the step calls.  No arithmetic of the method lives here;
every step runs in libbubblespec.so."""
import torch

from . import binding as B

TORCH_DTYPE = {B.BS_F32: torch.float32, B.BS_BF16: torch.bfloat16}


def fuse_weights(w, dtype, device):
    """Layout marshalling: per-matrix weights (oracle naming: wq/wk/wv, w_gate/w_up, ...) as torch tensors
    -> the fused row-major layout of bs_weights on `device`."""
    td = TORCH_DTYPE[dtype]
    dev = lambda t, dt=td: t.to(device=device, dtype=dt).contiguous()
    out = {"embed": dev(w["embed"]), "lm_head": dev(w["lm_head"]), "final_norm": dev(w["final_norm"], torch.float32),
           "attn_norm": [], "wqkv": [], "wo": [], "mlp_norm": [], "w_gate_up": [], "w_down": []}
    for lw in w["layers"]:
        out["attn_norm"].append(dev(lw["attn_norm"], torch.float32))
        out["mlp_norm"].append(dev(lw["mlp_norm"], torch.float32))
        out["wqkv"].append(torch.cat([dev(lw["wq"]), dev(lw["wk"]), dev(lw["wv"])], dim=0).contiguous())
        out["wo"].append(dev(lw["wo"]))
        out["w_gate_up"].append(torch.cat([dev(lw["w_gate"]), dev(lw["w_up"])], dim=0).contiguous())
        out["w_down"].append(dev(lw["w_down"]))
    return out


def page_table(n_slots, max_ctx, slot_tokens, page_perm_seed, device):
    """(block table [n_slots, most pages of a slot], number of pages): every slot gets the pages of max_ctx tokens, or of its own
    entry of slot_tokens (entries beyond a slot's pages are -1); page_perm_seed scatters the page ids."""
    P = B.BS_PAGE_TOKENS
    caps = [int(max_ctx)] * n_slots if slot_tokens is None else [int(t) for t in slot_tokens]
    assert len(caps) == n_slots
    pages_of = [(c + P - 1) // P for c in caps]
    n_pages = sum(pages_of)
    ids = torch.arange(n_pages, dtype=torch.int32)
    if page_perm_seed is not None:
        g = torch.Generator().manual_seed(page_perm_seed)
        ids = ids[torch.randperm(n_pages, generator=g)]
    table = torch.full((n_slots, max(pages_of)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages_of):
        table[b, :n] = ids[at:at + n]
        at += n
    return table.contiguous().to(device), n_pages


class Engine:
    """Owns the device buffers of one context and forwards to the C ABI."""

    def __init__(self, desc, weights, n_slots, max_ctx, B_max, k_max, device="cuda:0", page_perm_seed=None,
                 slot_tokens=None, kv_bits=16):
        """max_ctx: token capacity of every slot; slot_tokens (optional, one entry per slot) gives every slot its own
        capacity instead, so that a ragged batch only takes the pages it needs (block-table entries beyond a slot's
        pages are -1).  kv_bits = 8 (bf16 models): the cache holds 8 bits per element (KvqCache, bs_kvq_bind)."""
        if kv_bits not in (16, 8) or (kv_bits == 8 and desc["dtype"] != B.BS_BF16):
            raise B.BsError(B.BS_EINVAL, "kv_bits is 16 or, for bf16 models, 8")
        self.desc = dict(desc)
        self.device = torch.device(device)
        self.cdesc = B.make_desc(desc)
        self.B_max, self.k_max = B_max, k_max
        self.weights = weights
        # page encoding: float32 models store float32; bf16 models store bf16-rounded values as float16 bits
        td = torch.float32 if desc["dtype"] == B.BS_F32 else torch.float16
        P = B.BS_PAGE_TOKENS
        self.block_table, self.n_pages = page_table(n_slots, max_ctx, slot_tokens, page_perm_seed, self.device)
        self.max_pages = self.block_table.shape[1]
        self.n_slots = n_slots
        page_elems = desc["n_kv_heads"] * P * desc["head_dim"]
        self.kvq = None
        if kv_bits == 8:
            self.kvq = KvqCache(desc["n_layers"], desc["n_q_heads"], desc["n_kv_heads"], desc["head_dim"], n_slots, max_ctx, k_max + 1,
                                device=self.device, block_table=self.block_table, n_pages=self.n_pages, own_workspace=False)
            self.k_pages, self.v_pages = self.kvq.k_pages, self.kvq.v_pages
        else:
            # pages are zero-initialised: masked positions still enter the P*V product with weight 0
            self.k_pages = [torch.zeros(self.n_pages, page_elems, dtype=td, device=self.device)
                            for _ in range(desc["n_layers"])]
            self.v_pages = [torch.zeros(self.n_pages, page_elems, dtype=td, device=self.device)
                            for _ in range(desc["n_layers"])]
        self.ctx_len = torch.zeros(n_slots, dtype=torch.int32, device=self.device)
        nbytes = B.bs_workspace_bytes(self.cdesc, B_max, k_max)
        if nbytes == 0:
            raise B.BsError(B.BS_ESHAPE, "bs_workspace_bytes rejected the shape")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        kv = dict(n_pages=self.n_pages, n_slots=n_slots, max_pages_per_seq=self.max_pages, k_pages=self.k_pages,
                  v_pages=self.v_pages, block_table=self.block_table, ctx_len=self.ctx_len)
        self.ctx = B.bs_create(self.cdesc, weights, kv, self.workspace, B_max, k_max)
        if self.kvq is not None:
            self._kvq_workspace = torch.zeros(max(B.bs_kvq_bind_bytes(self.ctx), 1), dtype=torch.uint8, device=self.device)
            B.bs_kvq_bind(self.ctx, self.kvq.desc, self._kvq_workspace)
            self.kvq.workspace = self._kvq_workspace
        self._pool = None

    def close(self):
        if self.ctx is not None:
            B.bs_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- draft database -----------------------------------------------------------------------
    def pool_bind(self, pool_tokens, rollout_offsets, prompt_rollout_begin):
        self._pool = (pool_tokens.to(self.device, torch.int32).contiguous(),
                      rollout_offsets.to(self.device, torch.int64).contiguous(),
                      prompt_rollout_begin.to(self.device, torch.int32).contiguous())
        B.bs_pool_bind(self.ctx, self._pool[2].numel() - 1, self._pool[1].numel() - 1, *self._pool)

    def index_bind(self, blob_host):
        """Binds a prebuilt index (NumPy blob from binding.bs_index_build); None unbinds and returns to the scan."""
        if blob_host is None:
            self._index = None
            B.bs_index_bind(self.ctx, None, None)
            return
        self._index = (blob_host, torch.from_numpy(blob_host).to(self.device))
        B.bs_index_bind(self.ctx, *self._index)

    def draft_lookup(self, seq_prompt, tail_tokens, max_match, min_match, k_max):
        n = seq_prompt.numel()
        draft_tokens = torch.empty(n, max(k_max, 1), dtype=torch.int32, device=self.device)[:, :k_max].contiguous()
        draft_len = torch.empty(n, dtype=torch.int32, device=self.device)
        B.bs_draft_lookup(self.ctx, n, seq_prompt, tail_tokens, max_match, min_match, k_max, draft_tokens, draft_len)
        return draft_tokens, draft_len

    # -- step ---------------------------------------------------------------------------------
    def verify_step(self, seq_slot, last_token, draft_tokens, draft_len, k_max, want_logits=False):
        n = seq_slot.numel()
        logits = None
        if want_logits:
            logits = torch.zeros(n * (k_max + 1), self.desc["vocab"], dtype=torch.float32, device=self.device)
        B.bs_verify_step(self.ctx, n, seq_slot, last_token, draft_tokens, draft_len, k_max, logits)
        return logits

    def accept_resample(self, draft_tokens, draft_len, k_max, u_accept, u_sample, q_logits=None, temperature=1.0,
                        eos_id=-1, emit_bonus=True, logits=None, vocab=None):
        n = draft_len.numel()
        out = dict(n_accepted=torch.empty(n, dtype=torch.int32, device=self.device),
                   out_tokens=torch.empty(n, k_max + 1, dtype=torch.int32, device=self.device),
                   n_emitted=torch.empty(n, dtype=torch.int32, device=self.device),
                   near_tie=torch.empty(n, dtype=torch.int32, device=self.device))
        q_dtype = B.BS_F32
        if q_logits is not None:
            q_dtype = B.BS_BF16 if q_logits.dtype == torch.bfloat16 else B.BS_F32
        args = (draft_tokens, draft_len, k_max, q_logits, q_dtype, float(temperature), eos_id, emit_bonus, u_accept,
                u_sample, out["n_accepted"], out["out_tokens"], out["n_emitted"], out["near_tie"])
        if logits is None:
            B.bs_accept_resample(self.ctx, n, *args)
        else:
            B.bs_accept_resample_logits(self.ctx, n, vocab if vocab is not None else logits.shape[1], logits, *args)
        return out

    def set_filter(self, top_k=0, top_p=1.0):
        """Top-k / top-p filtering of the target distribution for the following accept steps (0 / 1.0: off).
        bf16 models get the float32 logits scratch the filtered path needs, allocated on first use."""
        on = top_k > 0 or top_p < 1.0
        if on and self.desc["dtype"] == B.BS_BF16 and getattr(self, "_filter_logits", None) is None:
            self._filter_logits = torch.empty(self.B_max * (self.k_max + 1), self.desc["vocab"], dtype=torch.float32,
                                              device=self.device)
        B.bs_set_filter(self.ctx, top_k, top_p, getattr(self, "_filter_logits", None) if on else None)

    def kv_commit(self, seq_slot, n_commit):
        B.bs_kv_commit(self.ctx, seq_slot.numel(), seq_slot, n_commit)

    def kv_lengths(self, seq_slot):
        out = torch.empty(seq_slot.numel(), dtype=torch.int32, device=self.device)
        B.bs_kv_lengths(self.ctx, seq_slot.numel(), seq_slot, out)
        return out

    def kv_write(self, layer, slot, pos0, k_rows, v_rows):
        B.bs_kv_write(self.ctx, layer, slot, pos0, k_rows.shape[0], k_rows.contiguous(), v_rows.contiguous())

    def kv_read(self, layer, slot, pos0, n):
        td = TORCH_DTYPE[self.desc["dtype"]]
        shape = (n, self.desc["n_kv_heads"], self.desc["head_dim"])
        k = torch.empty(shape, dtype=td, device=self.device)
        v = torch.empty(shape, dtype=td, device=self.device)
        B.bs_kv_read(self.ctx, layer, slot, pos0, n, k, v)
        return k, v

    def poll_status(self):
        return B.bs_poll_status(self.ctx)


class KvqCache:
    """Owns a KV cache in 8 bits (pages, scales and block table of every layer, attention workspace) and forwards to bs_kvq_*.
    Slots, capacities and page permutation as in Engine.  Rows are packed in batch order; n_max / q_max bound the rows of a
    sequence, which are on the device.  One attention call at a time: the workspace is shared (that of an Engine's cache with its verify
    steps).  `status` (one int32 on the device) collects BS_FAULT_* bits until poll_status."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, n_slots, max_ctx, q_max, device="cuda:0", page_perm_seed=None,
                 slot_tokens=None, block_table=None, n_pages=0, own_workspace=True):
        """block_table, n_pages: those of another owner (an Engine) instead of own ones, which sets `workspace` where own_workspace is False."""
        self.device = torch.device(device)
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.n_slots, self.q_max = n_q_heads, n_kv_heads, head_dim, n_slots, q_max
        self.block_table, self.n_pages = (block_table, n_pages) if block_table is not None else page_table(n_slots, max_ctx, slot_tokens, page_perm_seed, self.device)
        page = n_kv_heads * B.BS_PAGE_TOKENS * head_dim
        zeros = lambda *shape, dtype: [torch.zeros(*shape, dtype=dtype, device=self.device) for _ in range(n_layers)]
        # zero-filled: masked positions still enter the P*V product with weight 0
        self.k_pages, self.v_pages = zeros(self.n_pages, page, dtype=torch.uint8), zeros(self.n_pages, page, dtype=torch.uint8)
        self.k_scale, self.v_scale = zeros(self.n_pages, n_kv_heads, dtype=torch.float32), zeros(self.n_pages, n_kv_heads, dtype=torch.float32)
        self.desc = [B.make_kvq_desc(dict(n_pages=self.n_pages, n_slots=n_slots, max_pages_per_seq=self.block_table.shape[1], n_kv_heads=n_kv_heads,
                                          head_dim=head_dim, k_pages=self.k_pages[l], v_pages=self.v_pages[l], k_scale=self.k_scale[l],
                                          v_scale=self.v_scale[l], block_table=self.block_table)) for l in range(n_layers)]
        nbytes = B.bs_kvq_workspace_bytes(n_q_heads, n_kv_heads, head_dim, q_max)
        if nbytes == 0:
            raise B.BsError(B.BS_ESHAPE, "bs_kvq_workspace_bytes rejected the shape")
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device) if own_workspace else None
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)

    def write(self, layer, seq_slot, pos0, n_rows, n_max, k_rows, v_rows):
        """k_rows, v_rows: bf16 [rows, n_kv_heads, head_dim], to positions pos0[b] .. of slot seq_slot[b]."""
        B.bs_kvq_write(self.desc[layer], seq_slot.numel(), seq_slot, pos0, n_rows, n_max, k_rows, v_rows, self.status)

    def read(self, layer, seq_slot, pos0, n_rows, n_max, total):
        """The values held of `total` rows in all, bf16 [total, n_kv_heads, head_dim]."""
        k = torch.empty(total, self.n_kv_heads, self.head_dim, dtype=torch.bfloat16, device=self.device)
        v = torch.empty_like(k)
        B.bs_kvq_read(self.desc[layer], seq_slot.numel(), seq_slot, pos0, n_rows, n_max, k, v, self.status)
        return k, v

    def attention(self, layer, q, seq_slot, ctx_len, q_len, q_max, out=None):
        """q: bf16 [rows, n_q_heads, head_dim]; row i of sequence b sees positions 0 .. ctx_len[b] + i."""
        if q_max > self.q_max:
            raise B.BsError(B.BS_ECAPACITY, "KvqCache.attention: q_max exceeds that of the workspace")
        if self.workspace is None:
            raise B.BsError(B.BS_ESTATE, "KvqCache.attention: the cache was made without a workspace, and none has been set")
        if out is None:
            out = torch.empty(q.shape[0], self.n_q_heads, self.head_dim, dtype=torch.bfloat16, device=self.device)
        B.bs_kvq_attention(self.desc[layer], seq_slot.numel(), seq_slot, ctx_len, q_len, q_max, self.n_q_heads, q, out, self.workspace, self.status)
        return out

    def poll_status(self):
        fault = int(self.status.item())
        self.status.zero_()
        return fault


class LogprobScorer:
    """Owns the workspace of bs_token_logprobs for up to B_max sequences of k_max + 1 rows.  The tokens, counts and logits of an
    accept call can be passed on; `status` collects BS_FAULT_* bits until poll_status.  One call at a time: the workspace is shared.  The law is the softmax of
    the logits passed: for tokens sampled under Engine.set_filter the caller masks (-inf) what the filter dropped, else log p is that of the unfiltered law."""

    def __init__(self, B_max, k_max, vocab, n_top, device="cuda:0"):
        self.B_max, self.k_max, self.vocab, self.n_top = B_max, k_max, vocab, n_top
        self.device = torch.device(device)
        nbytes = B.bs_token_logprobs_workspace_bytes(B_max, k_max, vocab, n_top)
        if nbytes == 0:
            raise B.BsError(B.BS_ESHAPE, "bs_token_logprobs_workspace_bytes rejected the sizes")
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._index = self.workspace.get_device()
        self._workspace_at, self._workspace_bytes, self._status_at = self.workspace.data_ptr(), nbytes, self.status.data_ptr()

    def __call__(self, logits, tokens, n_tokens=None, draft_len=None, temperature=1.0):
        """logits [rows, vocab] (float32 or bf16, packed); tokens [B, k_max + 1]; n_tokens, draft_len [B] or None (all rows).
        Returns logprob, entropy [B, k_max + 1] and, with n_top, top_tokens, top_logprobs [B, k_max + 1, n_top]."""
        n, width = tokens.shape
        if n > self.B_max or width > self.k_max + 1 or logits.shape[1] != self.vocab:
            raise B.BsError(B.BS_ESHAPE, "LogprobScorer: sizes exceed those of the workspace")
        if logits.get_device() != self._index:
            raise B.BsError(B.BS_EINVAL, "LogprobScorer: logits on %s, workspace on %s" % (logits.device, self.device))
        lp = torch.empty((n, width), device=self.device)
        h = torch.empty_like(lp)
        out, at = {"logprob": lp, "entropy": h}, (None, None)
        if self.n_top:
            out["top_tokens"] = torch.empty((n, width, self.n_top), dtype=torch.int32, device=self.device)
            out["top_logprobs"] = torch.empty((n, width, self.n_top), device=self.device)
            at = out["top_tokens"].data_ptr(), out["top_logprobs"].data_ptr()
        # (addresses of what was just made need no checks)
        B.bs_token_logprobs(n, self.vocab, logits, draft_len, width - 1, tokens, n_tokens, temperature, self.n_top, lp.data_ptr(), h.data_ptr(), at[0], at[1],
                            self._workspace_at, self._status_at, self._workspace_bytes)
        return out

    def poll_status(self):
        fault = int(self.status.item())
        self.status.zero_()
        return fault
