"""The paged operators used together, as a serving program would: whole models run through sps_linear, sps_paged_append and
sps_paged_attention over a cache of scattered pages, several sequences of unlike lengths in one batch, against the oracle's
logits -- prompts, a scoring pass of K + 1 rows per sequence, a rollback (kv_len moved back, nothing copied), single tokens
drawn with sps_sample_filtered."""
import numpy as np
import pytest
import torch

import oracle
import paper_2302_01318_b200 as sps
import sps_synth
from gpu_util import oracle_model
from paged_util import BF16, DEV, F32, workspace

pytestmark = pytest.mark.gpu
TOL = {"tiny": 1e-3, "tiny_gqa": 1e-3, "tiny_bf16": 5e-2, "tiny_mqa_bf16": 5e-2}   # the handle's own logit tolerances


class PagedModel:
    """A decoder over paged caches: one cache per layer, one page table for all."""

    def __init__(self, cfg, w, n_pages, page):
        self.cfg, self.w = cfg, w
        self.H, self.Hkv, self.d = cfg["n_heads"], cfg["n_kv_heads"], cfg["d_head"]
        cdt = F32 if cfg["dtype"] == 0 else BF16
        self.caches = [sps.PagedCache(*(torch.full((n_pages, self.Hkv, page, self.d), float("nan"), dtype=cdt, device=DEV) for _ in "kv"))
                       for _ in range(cfg["n_layers"])]
        self.plan = sps.Rotary(torch.from_numpy(sps.sps_rotary_frequencies(self.d, cfg["rope_base"])).to(DEV))
        self.ws = workspace(self.caches[0], self.H, F32)

    def linear(self, W, X):
        dtype = 0 if W.dtype == F32 else 1
        out = torch.empty((X.shape[0], W.shape[0]), device=DEV)
        for r in range(0, X.shape[0], 16):
            x = X[r:r + 16].contiguous()
            y = torch.empty((x.shape[0], W.shape[0]), device=DEV)
            ws = torch.zeros(sps.sps_linear_workspace_bytes(dtype, x.shape[0], *W.shape), dtype=torch.uint8, device=DEV)
            sps.sps_linear(W, x, y, ws)
            out[r:r + 16] = y
        return out

    def norm(self, x, g):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.cfg["rms_eps"]) * g

    def forward(self, tokens, batch):
        x = self.w["tok_embed"][torch.as_tensor(tokens, device=DEV).long()].float()
        rows = x.shape[0]
        for lw, cache in zip(self.w["layers"], self.caches):
            h = self.norm(x, lw["attn_norm"])
            qkv = torch.cat([self.linear(lw[k], h) for k in ("wq", "wk", "wv")], 1).view(rows, self.H + 2 * self.Hkv, self.d)
            q, k, v = qkv[:, :self.H], qkv[:, self.H:self.H + self.Hkv], qkv[:, self.H + self.Hkv:]
            sps.sps_paged_append(cache, batch, k, v, self.plan, q, q)
            o = torch.empty((rows, self.H, self.d), device=DEV)
            sps.sps_paged_attention(cache, batch, q, o, self.ws)
            x = x + self.linear(lw["wo"], o.view(rows, -1))
            x = x + self.linear(lw["w_down"], torch.nn.functional.gelu(self.linear(lw["w_up"], self.norm(x, lw["ffn_norm"])), approximate="tanh"))
        return self.linear(self.w["unembed"], self.norm(x, self.w["final_norm"]))


@pytest.mark.parametrize("name", sorted(TOL))
def test_paged_model_matches_the_oracle(name):
    cfg = sps_synth.CONFIGS[name]["target"]
    w = sps_synth.make_weights(cfg, seed=3)
    V, page, n_pages = cfg["vocab"], 16, 24
    prompts = [list(map(int, sps_synth.make_prompt(i, n, V))) for i, n in enumerate((37, 5, 18))]
    model = PagedModel(cfg, sps_synth.weights_to(w, DEV), n_pages, page)
    free = list(torch.randperm(n_pages, generator=torch.Generator().manual_seed(0)).tolist())
    table = torch.zeros((3, 6), dtype=torch.int32)
    held = [0, 0, 0]

    def batch_for(news, lens):
        for b, L in enumerate(lens):
            while held[b] * page < L:
                table[b, held[b]] = free.pop()
                held[b] += 1
        q_start = torch.tensor([0] + list(news)).cumsum(0).to(torch.int32).to(DEV)
        return sps.PagedBatch(q_start, torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV), max_q=max(news))

    def want(seqs, news):
        out = []
        for s, n in zip(seqs, news):
            ref = oracle_model(cfg, w, 64)
            out.append(ref.forward64(np.array(s, dtype=np.int32), np.arange(len(s), dtype=np.int32))[len(s) - n:])
        return np.concatenate(out)

    def run(seqs, news):
        batch = batch_for(news, [len(s) for s in seqs])
        toks = [t for s, n in zip(seqs, news) for t in s[len(s) - n:]]
        logits = model.forward(toks, batch)
        assert int(batch.status) == 0
        assert np.abs(logits.double().cpu().numpy() - want(seqs, news)).max() < TOL[name]
        return logits

    run(prompts, [len(p) for p in prompts])                                          # prompts of unlike lengths in one pass
    drafts = [list(map(int, sps_synth.make_prompt(50 + i, 5, V))) for i in range(3)]
    run([p + d for p, d in zip(prompts, drafts)], [5, 5, 5])                         # scoring pass: K + 1 = 5 rows each
    seqs = [p + d[:k] for p, d, k in zip(prompts, drafts, (2, 5, 1))]                # 2, 5 and 1 kept: lengths move back
    seqs = [s + [7 + i] for i, s in enumerate(seqs)]
    for step in range(3):                                                            # one token each, greedy
        logits = run(seqs, [1, 1, 1])
        nxt = torch.zeros(3, dtype=torch.int32, device=DEV)
        sps.sps_sample_filtered(logits, 0.0, 0, 1.0, 0, step, 0, nxt)
        assert torch.equal(nxt.long(), logits.argmax(-1))
        seqs = [s + [int(t)] for s, t in zip(seqs, nxt)]
