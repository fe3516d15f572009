"""Greedy speculative decoding end to end on the GPU: the drafter's trees verified by a small
target whose layers run on the target-side operators (Sec. 2.4 of FastEagle, "Parallel
Verification" and "Update and Iterate"): attention alone with PyTorch's matrix products, or whole
layers on the dense operators. Random weights stand in for trained ones.

    python examples/verify_cycle.py [--cache f32|bf16|e4m3] [--target attention|layers] [--steps N]

prints the accepted tokens per cycle and checks that the text equals token-by-token decoding.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2509_20416_gb300 as fe  # noqa: E402
from fe_synth import workloads as wl  # noqa: E402


class ToyTarget:
    """Embedding, attention layers x += W_o attention(RMSNorm(x)), final norm and head. Rows are
    float32, or bfloat16 where the cache is 16- or 8-bit."""

    def __init__(self, cfg: dict, W: dict, cache: str, batch: int, max_seq: int, n_layers: int = 2, page_size: int = 16,
                 seed: int = 1):
        self.H, self.Hkv, self.hd, self.d = cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["d"]
        self.dt = torch.float32 if cache == "f32" else torch.bfloat16
        g = torch.Generator().manual_seed(seed)
        mat = lambda *s: (torch.randn(*s, generator=g) / s[-1] ** 0.5).to(self.dt).cuda()
        rows = (self.H + 2 * self.Hkv) * self.hd
        self.layers = [dict(qkv=mat(rows, self.d), o=mat(self.d, self.H * self.hd)) for _ in range(n_layers)]
        self.embed, self.head = (W[n].cuda().float() for n in ("embed", "lm_head"))
        self.t = fe.fe_target_init(dict(
            n_heads=self.H, n_kv_heads=self.Hkv, head_dim=self.hd, max_batch=batch, max_seq=max_seq, page_size=page_size,
            dtype="f32" if cache == "f32" else "bf16", cache_dtype=cache, rope_theta=cfg["rope_theta"]))
        pages = -(-max_seq // page_size)
        table = torch.randperm(batch * pages, generator=g).view(batch, pages).to(torch.int32).cuda()
        self.cache = fe.alloc_cache(self.t, n_layers, n_pages=batch * pages, page_table=table)

    def forward(self, tok, pos, start, n_rows=None, mask=None):
        """Tokens [B, T] at positions pos into slots start[b] + i; returns each one's next token and
        the drafter's features [B, T, 3 d] (the states before, between and after the layers)."""
        B, T = tok.shape
        x = self.embed[tok.long()] * 50.0
        states = [x]
        for i, L in enumerate(self.layers):
            u = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
            qkv = (u.to(self.dt) @ L["qkv"].T).view(B, T, self.H + 2 * self.Hkv, self.hd)
            q, k, v = qkv.split([self.H, self.Hkv, self.Hkv], 2)
            q = fe.fe_cache_write(self.t, self.cache, i, k, v, start, n_rows=n_rows, pos=pos, q=q)
            a, _ = fe.fe_tree_attention(self.t, self.cache, i, q, start, mask=mask, n_nodes=n_rows)
            x = x + (a.reshape(B, T, -1) @ L["o"].T).float()
            states.append(x)
        u = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
        feat = torch.cat([states[0], states[len(states) // 2], states[-1]], -1)
        return (u @ self.head.T).argmax(-1).to(torch.int32), feat


class LayerTarget(ToyTarget):
    """Whole layers: attention and a gated feed-forward block, each with a norm before it and the
    attention's with one behind it, and a head whose most probable token is the next."""

    def __init__(self, cfg: dict, W: dict, cache: str, batch: int, max_seq: int, n_layers: int = 2, page_size: int = 16,
                 seed: int = 1):
        super().__init__(cfg, W, cache, batch, max_seq, n_layers, page_size, seed)
        g = torch.Generator().manual_seed(seed + 1)
        mat = lambda *s: (torch.randn(*s, generator=g) / s[-1] ** 0.5).to(self.dt).cuda()
        gain = lambda: (1 + 0.1 * torch.randn(self.d, generator=g)).to(self.dt).cuda()
        for L in self.layers:
            L.update(attn_norm=gain(), post_norm=gain(), mlp_norm=gain(), gate=mat(cfg["ffn"], self.d), up=mat(cfg["ffn"], self.d),
                     down=mat(self.d, cfg["ffn"]))
        self.final_norm = gain()
        self.embed, self.head = self.embed.to(self.dt), self.head.to(self.dt)

    def forward(self, tok, pos, start, n_rows=None, mask=None):
        B, T = tok.shape
        t = self.t
        x = self.embed[tok.long()] * 50.0
        states = [x]
        for i, L in enumerate(self.layers):
            _, u = fe.fe_block_norm(t, x, pre_weight=L["attn_norm"])
            qkv = fe.fe_project(t, u, L["qkv"]).view(B, T, self.H + 2 * self.Hkv, self.hd)
            q, k, v = qkv.split([self.H, self.Hkv, self.Hkv], 2)
            q = fe.fe_cache_write(t, self.cache, i, k, v, start, n_rows=n_rows, pos=pos, q=q)
            a, _ = fe.fe_tree_attention(t, self.cache, i, q, start, mask=mask, n_nodes=n_rows)
            o = fe.fe_project(t, a.reshape(B, T, -1), L["o"])
            x, u = fe.fe_block_norm(t, x, o, post_weight=L["post_norm"], pre_weight=L["mlp_norm"])
            x = fe.fe_gated_ffn(t, u, L["gate"], L["up"], w_down=L["down"], residual=x)
            states.append(x)
        _, u = fe.fe_block_norm(t, x, pre_weight=self.final_norm)
        top = fe.fe_token_logprobs(t, fe.fe_project(t, u, self.head), top=1)[3]
        feat = torch.cat([states[0], states[len(states) // 2], states[-1]], -1).float()
        return top[..., 0].contiguous(), feat


TARGETS = {"attention": ToyTarget, "layers": LayerTarget}


def decode_plain(target: ToyTarget, prompts, steps: int):
    """Token by token: the prompt as one ragged chunk, then single-token decoding."""
    tok, n = pad(prompts)
    B, T = tok.shape
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    nxt, _ = target.forward(tok, torch.arange(T, dtype=torch.int32, device="cuda").repeat(B, 1), zero, n_rows=n)
    cur = nxt.gather(1, n.long()[:, None] - 1)
    out, at = [cur], n.clone()
    for _ in range(steps - 1):
        cur, _ = target.forward(cur.contiguous(), at[:, None].contiguous(), at)
        out.append(cur)
        at = at + 1
    return torch.cat(out, 1)


def pad(prompts):
    n = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
    tok = torch.zeros(len(prompts), max(len(p) for p in prompts), dtype=torch.int32)
    for b, p in enumerate(prompts):
        tok[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    return tok.cuda(), n


def decode_drafted(target: ToyTarget, h, cfg: dict, prompts, steps: int, top_k: int = 4, forced=None):
    """Cycles of draft, tree, target pass, verification and update. `forced` [B, steps] plants the
    known continuation among each level's candidates (random weights never agree by themselves).
    Returns the emitted tokens and the number accepted in each cycle."""
    N = cfg["n_layers"]
    tok, n = pad(prompts)
    B, Tp = tok.shape
    dev = "cuda"
    zero = torch.zeros(B, dtype=torch.int32, device=dev)
    kc = [torch.zeros(B, cfg["n_kv_heads"], cfg["max_seq"], cfg["head_dim"], device=dev) for _ in range(N)]
    vc = [torch.zeros_like(k) for k in kc]
    nxt, feat = target.forward(tok, torch.arange(Tp, dtype=torch.int32, device=dev).repeat(B, 1), zero, n_rows=n)
    # the drafter's rows of the prompt: position p from the features of p - 1 and the token at p
    before = torch.cat([torch.zeros_like(feat[:, :1]), feat[:, :-1]], 1)
    for p in range(0, Tp, N):
        L = min(N, Tp - p)
        fe.fe_commit(h, before[:, p:p + L].contiguous(), tok[:, p:p + L].contiguous(), (n - p).clamp(0, L),
                     torch.minimum(n, zero + p), kc, vc)
    last = n.long() - 1
    cur, f = nxt.gather(1, last[:, None])[:, 0].contiguous(), feat[torch.arange(B), last].contiguous()
    P = n.clone()
    text = [[int(c)] for c in cur]
    accepted = []
    while min(len(t) for t in text) < steps:
        out = fe.fe_draft_forward(h, f, cur, P, kc, vc, top_k)
        ids = out["topk_id"]
        if forced is not None:
            for b in range(B):
                for i in range(N):
                    at = len(text[b]) + i
                    if at < forced.shape[1] and (at + b) % 5:  # (some levels are left to the drafter's luck)
                        ids[b, i, 0 if (at + b) % 3 else top_k - 1] = forced[b, at]
        tree = fe.fe_build_tree(h, cur, ids, top_k)
        pos = P[:, None] + tree["depth"]
        nxt, feat = target.forward(tree["tok"], pos.contiguous(), P, mask=tree["mask"])
        v = fe.fe_verify_greedy(h, P, tree, nxt, top_k)
        fe.fe_cache_keep(target.t, target.cache, v["path"], v["n_accept"], P)
        # the drafter's rows of the accepted tokens: features of the node before, token of the node
        path = v["path"].long().clamp(min=0)
        prev = torch.cat([torch.zeros_like(path[:, :1]), path[:, :-1]], 1)
        take = lambda x, i: x.gather(1, i[..., None].expand(-1, -1, x.shape[-1]))
        fe.fe_commit(h, take(feat, prev).contiguous(), tree["tok"].gather(1, path), v["n_accept"], P + 1, kc, vc)
        acc = v["n_accept"].tolist()
        accepted.append(acc)
        for b in range(B):
            text[b] += tree["tok"][b, v["path"][b, :acc[b]].long()].tolist() + [int(v["bonus"][b])]
        end = torch.where(v["n_accept"] > 0, path.gather(1, (v["n_accept"].long() - 1).clamp(min=0)[:, None])[:, 0], 0)
        f, cur, P = feat[torch.arange(B), end].contiguous(), v["bonus"].clone(), P + 1 + v["n_accept"]
    for code in (fe.fe_last_device_status(h), fe.fe_target_status(target.t)):
        if code != fe.FE_OK:
            raise fe.FeError(code, "verification cycle")
    return [t[:steps] for t in text], accepted


def run(cache: str = "f32", steps: int = 24, batch: int = 3, seed: int = 0, target: str = "attention"):
    """Both decodings on fresh caches; returns (drafted text, plain text, accepted per cycle)."""
    make = TARGETS[target]
    cfg = wl.make_config("tiny", B=batch, max_seq=128)
    W = wl.make_weights(cfg)
    h = fe.fe_draft_init(dict(cfg, max_batch=batch), W)
    g = torch.Generator().manual_seed(seed)
    prompts = [torch.randint(0, cfg["vocab"], (5 + 4 * b,), generator=g).tolist() for b in range(batch)]
    plain = decode_plain(make(cfg, W, cache, batch, 128), prompts, steps)
    text, accepted = decode_drafted(make(cfg, W, cache, batch, 128), h, cfg, prompts, steps, forced=plain)
    return text, plain.tolist(), accepted


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", default="f32", choices=["f32", "bf16", "e4m3"])
    ap.add_argument("--target", default="attention", choices=list(TARGETS))
    ap.add_argument("--steps", type=int, default=24)
    a = ap.parse_args()
    text, plain, accepted = run(a.cache, a.steps, target=a.target)
    print("accepted per cycle:", accepted)
    print("equal to token-by-token decoding:", text == plain)


if __name__ == "__main__":
    main()
