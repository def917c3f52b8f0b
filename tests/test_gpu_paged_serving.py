"""A decode loop over a paged cache, as a server would write it: prompts prefilled together, their caches written into
pages, then single-token steps through the library's single steps, every token chosen by pp_sample; a sequence
that is done leaves its slot and its pages to the next prompt.

* float32 pages: the logits of every step against the oracle's on the same tokens (2e-2 max, 2e-3 mean, as for
  pp_generate), greedy tokens where the oracle's choice is clear.
* bf16 pages: each logits tensor within twice the error of an ideal bf16 pipeline (the oracle with every stored value
  rounded): both make the same roundings, of values that differ in their last bits.
* all pages, 8-bit ones too: every attention of the loop against float64 on what the pages hold, every token
  against pp_sample's definition on the loop's own logits."""
import numpy as np
import pytest
import torch

from oracle import decoder as D
from oracle import generate as G
from paper_2404_09529_amd import prepack as pp
from paper_2404_09529_amd import workloads as W

from .gpu_util import bf16_dev, f32_dev, host64, i32_dev, oracle_weights, require_gpu
from .test_gpu_paged import PAGES, Pool, check_attention
from .test_gpu_sample import definition

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Server:
    """k slots over pools of one page table; free pages are handed out from a list, the last freed first."""

    def __init__(self, case, lm_head, kv, k, page, max_pages, n_pages):
        self.case, self.k, self.page = case, k, page
        self.model = pp.DeviceModel(case.shape, case.weights)
        s = self.s = case.shape
        self.t = self.model.torch_dtype
        self.lm = bf16_dev(lm_head) if s.dtype == "bf16" else f32_dev(lm_head)
        self.table = np.full((k, max_pages), -1, dtype=np.int32)
        self.table_dev = i32_dev(self.table)
        self.free = list(range(n_pages))[::-1]
        self.pools = []
        for _ in range(s.n_layers):
            p = Pool.__new__(Pool)                    # for check_attention: its table is the server's
            p.kv, p.Hkv, p.D, p.page = kv, s.n_kv_heads, s.head_dim, page
            size = (n_pages, page, s.n_kv_heads * s.head_dim)
            p.k, p.v = (torch.full(size, 77, dtype=PAGES[kv][1]) for _ in range(2))
            p.ks, p.vs = (torch.full((n_pages, page, s.n_kv_heads), float("nan")) if kv == "i8" else None for _ in range(2))
            p.dev = {n: None if getattr(p, n) is None else getattr(p, n).cuda() for n in ("k", "v", "ks", "vs")}
            p.cache = pp.PagedCache(PAGES[kv][0], self.table_dev, *(p.dev[n] for n in ("k", "v", "ks", "vs")))
            self.pools.append(p)
        w = (s.n_heads + 2 * s.n_kv_heads) * s.head_dim
        empty = lambda n, dt=None: torch.empty((k, n), dtype=dt or self.t, device="cuda")
        self.x, self.logits = empty(s.d_model, torch.float32), empty(s.vocab, torch.float32)
        self.xn, self.qkv, self.out = empty(s.d_model), empty(w), empty(s.n_heads * s.head_dim)
        self.up, self.h = empty(2 * s.ffn_dim), empty(s.ffn_dim)
        self.lens = torch.zeros(k, dtype=torch.int32, device="cuda")
        self.tokens = torch.zeros(k, dtype=torch.int32, device="cuda")
        self.prob = torch.zeros(k, device="cuda")
        need = max(pp.pp_paged_attention_workspace_size(self.model.config, self.pools[0].cache), pp.pp_sample_workspace_size(k, s.vocab), 1)
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")   # calls of one stream share it

    def reserve(self, slot, tokens):
        """Pages for a slot's next tokens."""
        for j in range(-(-tokens // self.page)):
            if self.table[slot, j] < 0:
                self.table[slot, j] = self.free.pop()
        self.table_dev.copy_(torch.from_numpy(self.table))

    def release(self, slot):
        self.free += [int(p) for p in self.table[slot] if p >= 0]
        self.table[slot] = -1
        self.table_dev.copy_(torch.from_numpy(self.table))

    def enter(self, pre, pairs):
        """(prompt, slot) pairs: the prefill's rows into the slots' pages."""
        off = pre.dplan.plan.prompt_kv_off
        for prompt, slot in pairs:
            n = int(self.case.lengths[prompt])
            self.reserve(slot, n)
            seq, pos = torch.full((n,), slot, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
            kvw = pre.k_cache.shape[2]
            for l, p in enumerate(self.pools):
                a = int(off[prompt])
                pp.pp_paged_write(self.model.config, p.cache, seq, pos, n, pre.k_cache[l, a:a + n], kvw, pre.v_cache[l, a:a + n], kvw)

    def gemm(self, epilogue, a, b, c):
        d = a.shape[1]
        pp.pp_gemm(self.model.dtype_code, epilogue, a, d, b, d, c, c.shape[1], self.k, b.shape[0], d)

    def step(self, lens):
        """One token of every slot with lens[i] > 0 (that token included); self.tokens are fed."""
        s, m, code = self.s, self.model, self.model.dtype_code
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        self.x.copy_(m.embed[self.tokens.long().clamp(min=0)])
        for L, p in zip(m.layers, self.pools):
            pp.pp_rmsnorm(code, self.x, L["attn_norm"], self.k, s.d_model, s.rms_eps, self.xn)
            self.gemm(pp.PP_EPI_STORE, self.xn, L["wqkv"], self.qkv)
            w = self.qkv.shape[1]
            pp.pp_paged_append(m.config, p.cache, self.lens, self.qkv, w, self.qkv, w)     # the query stays in its place
            pp.pp_paged_attention(m.config, p.cache, self.lens, self.qkv, w, self.out, self.ws)
            p.table = torch.from_numpy(self.table)
            q = self.qkv.cpu().double()[:, :self.out.shape[1]].reshape(self.k, s.n_heads, s.head_dim)
            check_attention(self.out, q, p, lens, s.n_heads, s.dtype)
            self.gemm(pp.PP_EPI_RESIDUAL, self.out, L["wo"], self.x)
            pp.pp_rmsnorm(code, self.x, L["mlp_norm"], self.k, s.d_model, s.rms_eps, self.xn)
            if s.dtype == "bf16":
                self.gemm(pp.PP_EPI_SWIGLU, self.xn, L["w_gateup"], self.h)
            else:
                self.gemm(pp.PP_EPI_STORE, self.xn, L["w_gateup"], self.up)
                y = self.up.view(self.k, s.ffn_dim // 16, 2, 16)                           # 16 gate columns, 16 of up
                self.h.copy_((torch.nn.functional.silu(y[:, :, 0]) * y[:, :, 1]).reshape(self.k, -1))
            self.gemm(pp.PP_EPI_RESIDUAL, self.h, L["w_down"], self.x)
        pp.pp_rmsnorm(code, self.x, m.final_norm, self.k, s.d_model, s.rms_eps, self.xn)
        self.logits.copy_(self.xn.float() @ self.lm.float().t())

    def sample(self, settings, u):
        dev = {n: torch.tensor([x[n] for x in settings], dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda")
               for n in settings[0]}
        pp.pp_sample(self.logits, self.logits.shape[1], self.k, self.s.vocab, dev["t"], dev["top_k"], dev["top_p"], dev["min_p"],
                     torch.tensor(u, device="cuda"), self.tokens, self.ws, self.prob)
        return self.tokens.cpu().tolist()


SETTINGS = [dict(t=0.0, top_k=0, top_p=1.0, min_p=0.0), dict(t=0.7, top_k=40, top_p=0.9, min_p=0.0),
            dict(t=0.0, top_k=0, top_p=1.0, min_p=0.0), dict(t=1.3, top_k=0, top_p=1.0, min_p=0.02)]


def serve(dtype, kv, heads, new=6):
    """Five prompts through three slots; (prompt, tokens, logits) of each in the order that they end."""
    lengths = [5, 1, 17, 40, 9]
    H, Hkv = heads
    dims = dict(n_heads=H, n_kv_heads=Hkv) if dtype == "f32" else dict(d_model=512, n_heads=H, n_kv_heads=Hkv, ffn_dim=768, vocab=2000)
    case = W.make_case(1 if dtype == "f32" else 6, 3, n_layers=2, lengths=lengths, random_gains=True, **dims)
    lm_head = W.draw_lm_head(case.wl, 3, case.shape)
    server = Server(case, lm_head, kv, 3, 4, 16, 40)
    pre = pp.Prefill(server.model, pp.DevicePlan(pp.pp_pack(lengths, 0)))
    pre(i32_dev(case.tokens))
    firsts = torch.empty(5, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(pp.pp_first_token_workspace_size(server.model.config, pre.dplan), 1), dtype=torch.uint8, device="cuda")
    pp.pp_first_token(server.model.config, pre.dplan, pre.hidden, server.lm, ws, firsts)
    first = firsts.cpu().tolist()
    rng = np.random.default_rng(5)
    slots, waiting, done, steps = [None] * 3, [0, 1, 2, 3, 4], [], 0
    while waiting or any(slots):
        for i in range(3):
            if slots[i] is None and waiting and (i < 2 or steps):      # slot 2 is empty in the first step
                p = waiting.pop(0)
                server.enter(pre, [(p, i)])
                slots[i] = dict(prompt=p, fed=[], logits=[], next=first[p])
                server.tokens[i] = first[p]
        lens = [0 if s is None else lengths[s["prompt"]] + len(s["fed"]) + 1 for s in slots]
        for i, n in enumerate(lens):
            if n:
                server.reserve(i, n)
        server.step(lens)
        steps += 1
        u = rng.random(3).astype(np.float32).tolist()
        settings = [SETTINGS[0 if s is None else s["prompt"] % 4] for s in slots]
        tokens = server.sample(settings, u)
        logits = server.logits.cpu().numpy().copy()
        for i, s in enumerate(slots):
            if s is None:
                continue
            want, _, near = definition(logits[i], u=u[i], **settings[i])
            assert near or tokens[i] == want
            s["fed"].append(s["next"])
            s["logits"].append(logits[i])
            s["next"] = tokens[i]
            if len(s["fed"]) == new + s["prompt"]:
                done.append(s)
                server.release(i)
                slots[i] = None
    assert len(server.free) == 40
    return case, lm_head, done


@pytest.mark.parametrize("dtype,kv,heads", [("f32", "f32", (4, 4)), ("f32", "f32", (4, 2)), ("bf16", "bf16", (4, 2))])
def test_serving_matches_the_oracle(dtype, kv, heads):
    case, lm_head, done = serve(dtype, kv, heads)
    sh, w64, lm64 = D.Shape.of(case.shape), oracle_weights(case.weights), lm_head.astype(np.float64)
    off = np.concatenate([[0], np.cumsum(case.lengths)])
    assert sorted(s["prompt"] for s in done) == [0, 1, 2, 3, 4]
    for s in done:
        p = case.tokens[off[s["prompt"]]:off[s["prompt"] + 1]]
        ref = G.teacher_forced(p, s["fed"], w64, sh, lm64)
        got, want = np.stack(s["logits"]), np.stack(ref.logits)
        mx, mean = D.errors(got, want)
        if dtype == "f32":
            print(f"[serving] prompt {s['prompt']}: max {mx:.2e} mean {mean:.2e}", flush=True)
            assert mx <= 2e-2 and mean <= 2e-3
            if s["prompt"] % 2 == 0:                       # greedy
                chosen = s["fed"][1:] + [s["next"]]
                for t, row in enumerate(want):
                    top = np.sort(row)
                    assert top[-1] - top[-2] <= 1e-3 or chosen[t] == int(row.argmax())
        else:
            fmx, fmean = D.errors(np.stack(G.teacher_forced(p, s["fed"], w64, sh, lm64, rnd=D.round_bf16).logits), want)
            print(f"[serving] prompt {s['prompt']}: max {mx:.2e} mean {mean:.2e}, ideal bf16 {fmx:.2e} {fmean:.2e}", flush=True)
            assert mx <= 2 * fmx and mean <= 2 * fmean


@pytest.mark.parametrize("dtype,heads", [("f32", (4, 2)), ("bf16", (4, 1))])
def test_serving_from_8_bit_pages(dtype, heads):
    serve(dtype, "i8", heads)
