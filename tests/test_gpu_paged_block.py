"""A decoder block answered from the paged cache, step by step through the public calls, against the same weights in lr_block_fwd."""
import pytest
import torch

import synth_inputs as si
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HD, EPS = 128, 1e-5


def test_block_from_the_cache_is_the_block():
    """Two prompts in chunks, then single tokens: the rows of the block's output over the whole sequences.

    Bound: both sides are bf16 pipelines of the same data flow.  Each rounds q, k, v, the probabilities, o, z_o, y_o, h1, z_gu, g, u, m, z_d, y_d
    and y, sixteen tensors or fewer, by at most half a step, 2^-8 of an element; evenly spread that is 2^-8 / sqrt(3) of a tensor's norm, at random
    from tensor to tensor sqrt(16) times that for each side, 2^-8 * 4 / sqrt(3) * sqrt(2) < 2^-6.  (A norm, a SiLU's slope of at most 1.1 and
    a residual sum hand a relative error on without making it larger than that.)"""
    Bn, S, H, f, r, page = 2, 96, 4, 344, 64, 16
    d, f_ld = HD * H, si.pad_ld(f, 8)
    case = si.block_case(Bn, S, d, H, HD, f, r, seed=43)
    p = {k: v.to(DEV) for k, v in si.pack_block_params(case["params"], f, f_ld).items()}
    x = case["x"].to(DEV)
    tables = B.lr_rope_table(S, HD, device=DEV)
    desc = B.make_block_desc(Bn, S, d, H, HD, f, f_ld, r, eps=EPS, rope=tables)
    want, _ = B.lr_block_fwd(desc, p, x)

    def block(x, cache):
        _, _, (q, k, v) = B.lr_group_fwd(x, p["gamma1"], EPS, B.LR_NORM_ONLINE, p["w_dn_qkv"], p["w_up_qkv"].view(3, d, r))
        q = B.lr_kv_append(k, v, rope=tables, q=q, H=H, **cache)
        o, _ = B.lr_attention_paged_fwd(q, H=H, **cache)
        h1 = x + B.lr_linear_fwd(o, p["w_dn_o"], p["w_up_o"])[1]
        _, _, (gate, up) = B.lr_group_fwd(h1, p["gamma2"], EPS, B.LR_NORM_ONLINE, p["w_dn_gu"], p["w_up_gu"])
        return h1 + B.lr_linear_fwd(B.lr_swiglu_fwd(gate, up), p["w_dn_d"], p["w_up_d"])[1]

    g = torch.Generator(device=DEV).manual_seed(4)
    cache = {"k_cache": torch.full((16, page, H, HD), float("nan"), dtype=torch.bfloat16, device=DEV)}
    cache["v_cache"] = cache["k_cache"].clone()
    cache["page_table"] = torch.randperm(16, generator=g, device=DEV)[:12].to(torch.int32).view(2, 6).contiguous()
    rows, got, at = x.view(Bn, S, d), torch.empty_like(x).view(Bn, S, d), [0, 0]
    for steps in ((40, 1), (17, 60), (38, 33), (1, 1), (0, 1)):
        new = [slice(a, a + n) for a, n in zip(at, steps)]
        at = [a + n for a, n in zip(at, steps)]
        lens = {"cu_q": torch.tensor([0, steps[0], sum(steps)], dtype=torch.int32, device=DEV), "kv_len": torch.tensor(at, dtype=torch.int32, device=DEV)}
        y = block(torch.cat([rows[b, s] for b, s in enumerate(new)]), {**cache, **lens})
        got[0, new[0]], got[1, new[1]] = y[:steps[0]], y[steps[0]:]
    assert at == [S, S]
    torch.cuda.synchronize()
    diff = (got.view_as(want).float() - want.float()).norm() / want.float().norm()
    print(f"block from the cache: {float(diff):.2e} of the norm", flush=True)
    assert float(diff) < 2.0 ** -6
