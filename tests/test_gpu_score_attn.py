"""Attention with terms in its scores on the GPU against the fp64 oracle.

Tolerances, per element. h = half a step of the type relative to the value (bf16 2^-8,
fp32 2^-24), f = 2^-24.

- Scores carry f (head_dim + 8) (scale sum |q| |k| + |s|) from the products' sums, the
  cap, the bias and the base-2 exponential; this is the relative error of P, and of lse
  the absolute one, with what a sum over n keys adds, f n.  Call it r (over a row).
- o: P rounded to the type before the product (h sum P |v|), the result (h |o|), and r
  and the product's own sum, (r + f n) sum P |v|.
- dv likewise; dq, dk: P (dP - delta) rounded (h) before the product, and the row term
  from o as it is kept: an error of delta by sum |d_o| (h |o| + (h + r) sum P |v|).
- dtable: fp32 throughout, the row term too: f (head_dim + 16 + n) of the sums of the
  magnitudes that enter it.
"""
import numpy as np
import pytest

from oracle import score_oracle as so

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Case:
    def __init__(self, dtype="bf16", batch=1, seq=64, heads=2, kv_heads=None, d=64, seq_q=None,
                 causal=True, window=None, cap=0.0, slopes=False, buckets=0, max_distance=0,
                 docs=None, prefix=None, pad=64, q_std=2.0, seed=0):
        import torch
        from paper_2402_15627_amd import pblock as pb
        self.dtype, self.pb = dtype, pb
        kv_heads = kv_heads or heads
        seq_q = seq_q or seq
        window = window or seq
        act = torch_type(dtype)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.empty(s, device="cuda").normal_(generator=g)  # noqa: E731
        self.shape = (batch, seq_q, seq, heads, kv_heads, d)
        self.q = (rnd(batch * seq_q, heads * d + pad) * q_std).to(act)[:, :heads * d]
        kv = rnd(batch * seq, 2 * kv_heads * d + pad).to(act)
        self.k, self.v = kv[:, :kv_heads * d], kv[:, kv_heads * d:2 * kv_heads * d]
        self.d_o = rnd(batch * seq_q, heads * d + 2 * pad).to(act)[:, :heads * d]
        ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.t = dict(docs=ints(docs), prefix=ints(prefix),
                      slopes=torch.exp2(-torch.arange(1, heads + 1, device="cuda") * 4.0 / heads)
                      if slopes else None, table=rnd(buckets, heads) if buckets else None)
        self.cfg = pb.score_attn_config(batch, seq_q, seq, heads, kv_heads, d, causal, window,
                                        cap=cap, buckets=buckets, max_distance=max_distance,
                                        dtype=dtype)
        self.see = so.visible(batch, seq_q, seq, causal, window, docs, prefix)
        self.terms = dict(cap=cap, causal=causal, max_distance=max_distance)
        for n in ("slopes", "table"):
            if self.t[n] is not None:
                self.terms[n] = self.t[n].double().cpu().numpy()
        new = lambda rows, width: torch.full((rows, width + pad), 7.0, dtype=act, device="cuda")  # noqa: E731
        self.full = dict(o=new(batch * seq_q, heads * d), dq=new(batch * seq_q, heads * d),
                         dkv=new(batch * seq, 2 * kv_heads * d))
        self.o, self.dq = self.full["o"][:, :heads * d], self.full["dq"][:, :heads * d]
        self.dk = self.full["dkv"][:, :kv_heads * d]
        self.dv = self.full["dkv"][:, kv_heads * d:2 * kv_heads * d]
        self.lse = torch.full((batch, heads, seq_q), 7.0, device="cuda")
        self.dtable = torch.full((buckets, heads), 7.0, device="cuda") if buckets else None
        self.pad = pad

    def ws(self, mode):
        import torch
        n = self.pb.pblock_score_attn_workspace_bytes(self.cfg, mode)
        return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") if n else None

    def forward(self, split=True, stream=None, ws=None):
        ws = self.ws(self.pb.ATTN_WS_FORWARD) if split and ws is None else ws
        self.pb.pblock_score_attn_forward(self.cfg, self.q, self.k, self.v, self.o, self.lse,
                                          ws=ws, stream=stream, **self.t)

    def backward(self, mode=None, stream=None, ws=None):
        ws = self.ws(self.pb.ATTN_WS_BACKWARD if mode is None else mode) if ws is None else ws
        self.pb.pblock_score_attn_backward(self.cfg, self.q, self.k, self.v, self.o, self.d_o,
                                           self.lse, self.dq, self.dk, self.dv, ws,
                                           dtable=self.dtable, stream=stream, **self.t)

    def numpy(self, x, kv=False):
        b, sq, sk, h, kvh, d = self.shape
        return x.double().cpu().numpy().reshape(b, sk if kv else sq, kvh if kv else h, d)

    def oracle(self):
        d = self.shape[-1]
        return so.attention(self.numpy(self.q), self.numpy(self.k, True), self.numpy(self.v, True),
                            self.see, float(np.float32(d ** -0.5)), d_o=self.numpy(self.d_o),
                            **self.terms)

    def check(self, r, names):
        import torch
        d, seq = self.shape[-1], self.shape[2]
        h = 2.0 ** -8 if self.dtype == "bf16" else F
        rel = F * (d + 8) * float(r["a_s"].max(initial=0.0)) + F * seq
        got = dict(o=self.numpy(self.o), dq=self.numpy(self.dq), dk=self.numpy(self.dk, True),
                   dv=self.numpy(self.dv, True), lse=self.lse.double().cpu().numpy())
        tol = dict(o=h * (r["a_o"] + abs(r["o"])) + rel * r["a_o"],
                   dv=h * (r["a_dv"] + abs(r["dv"])) + rel * r["a_dv"],
                   dq=h * (r["a_dq"] + abs(r["dq"])) + 2 * rel * r["a_dq"] + (h + rel) * r["e_dq"],
                   dk=h * (r["a_dk"] + abs(r["dk"])) + 2 * rel * r["a_dk"] + (h + rel) * r["e_dk"],
                   lse=rel + F * abs(np.where(np.isfinite(r["lse"]), r["lse"], 0.0)))
        if self.dtable is not None:
            got["dtable"] = self.dtable.double().cpu().numpy()
            if "dtable" in r:
                tol["dtable"] = F * (d + 16 + seq) * r["a_dtable"]
        for n in names:
            if n not in got:
                continue
            a, w = got[n], r[n]
            fine = np.isfinite(w)
            assert np.array_equal(a[~fine], w[~fine]), n
            off = abs(a - w)[fine] - 1.02 * tol[n][fine] - 1e-30
            assert np.isfinite(a[fine]).all(), n
            assert (off <= 0).all(), (n, float(off.max()), float(abs(a - w)[fine].max()))
        for n, x in self.full.items():
            if (n == "o") == ("o" in names):
                assert bool((x[:, -self.pad:] == 7.0).all()), n

    def run(self):
        import torch
        self.forward()
        torch.cuda.synchronize()
        r = self.oracle()
        self.check(r, ("o", "lse"))
        self.backward()
        torch.cuda.synchronize()
        self.check(r, ("dq", "dk", "dv", "dtable"))
        return r


# every term alone and together, odd sizes, shared heads, each head width and type
CASES = {
    "plain": dict(seq=130, heads=2),
    "one": dict(seq=1, heads=1),
    "one_biased": dict(seq=1, heads=2, kv_heads=1, cap=5.0, buckets=8, max_distance=16),
    "two": dict(batch=2, seq=2, heads=1, d=96, slopes=True),
    "window": dict(seq=200, window=70, d=96),
    "window_1": dict(seq=70, window=1),
    "both_ways": dict(seq=150, causal=False),
    "both_ways_window": dict(batch=2, seq=193, causal=False, window=33, d=128, slopes=True),
    "cap": dict(seq=140, cap=3.0, d=128),
    "cap_large": dict(seq=65, cap=50.0, q_std=8.0),
    "slopes": dict(seq=129, heads=3, slopes=True),
    "group_2": dict(seq=100, heads=4, kv_heads=2, slopes=True),
    "group_5": dict(seq=90, heads=5, kv_heads=1, d=96, cap=10.0),
    "group_8": dict(batch=2, seq=77, heads=16, kv_heads=2, slopes=True),
    "group_3_buckets": dict(seq=150, heads=6, kv_heads=2, buckets=16, max_distance=40),
    "buckets": dict(seq=300, heads=2, buckets=32, max_distance=128),
    "buckets_both": dict(seq=300, heads=2, buckets=32, max_distance=64, causal=False),
    "buckets_few": dict(seq=100, heads=2, buckets=2, max_distance=5),
    "buckets_many": dict(seq=180, heads=2, buckets=64, max_distance=64, d=128),
    "buckets_far": dict(seq=200, heads=1, buckets=8, max_distance=100000),
    "buckets_all": dict(batch=2, seq=170, heads=4, kv_heads=1, buckets=32, max_distance=50, cap=8.0,
                        docs=[3, 60, 60, 171, 333], prefix=[9, 4, 100, 20], d=96),
    "docs": dict(batch=2, seq=100, docs=[0, 31, 32, 97, 140, 200]),
    "docs_padding": dict(seq=300, docs=[5, 100, 131], heads=2),
    "docs_none": dict(seq=70, docs=[0]),
    "docs_ones": dict(seq=70, docs=list(range(71))),
    "docs_beyond": dict(seq=64, docs=[-5, 20, 1000]),
    "prefix": dict(batch=2, seq=140, prefix=[70, 0], window=20),
    "prefix_docs": dict(seq=260, docs=[0, 100, 260], prefix=[64, 300], window=16, slopes=True),
    "prefix_both_ways": dict(seq=130, causal=False, window=5, prefix=[40]),
    "token": dict(batch=3, seq=150, seq_q=1, heads=8, kv_heads=2, slopes=True),
    "token_docs": dict(batch=2, seq=90, seq_q=1, docs=[0, 90, 170, 180], buckets=8, max_distance=20),
    "last_queries": dict(batch=2, seq=140, seq_q=37, heads=4, kv_heads=2, window=50, cap=4.0),
    "last_queries_prefix": dict(batch=2, seq=100, seq_q=10, causal=False, window=9, prefix=[3, 99]),
    "long_row": dict(seq=700, heads=1, slopes=True, d=128),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_score_attn(name, dtype):
    print(name, dtype, flush=True)
    Case(dtype=dtype, **CASES[name]).run()
