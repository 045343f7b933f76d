"""Scored routing and 8-bit experts together, as a program uses them: weights
quantised and packed, whole passes of Algorithm 1 by the Python driver and by
the library (host- and device-scheduled).  Each stage of a pass against the
oracle on the GPU's own inputs, and the same bits from every driver and policy."""
import numpy as np
import pytest
import torch

from oracle import experts8 as o8
from oracle import permute as operm
from test_gpu_experts8 import F8, Case, to64

pytestmark = pytest.mark.gpu


def make(dtype, H, F, E, k, S, L, N, T, *, router=True, balance=True, seed=0, D=2):
    """(stack, start, bf16 or fp32 weights of each layer, router arguments)."""
    from paper_2608_07964_amd import binding as B
    from paper_2608_07964_amd.driver import Stack, pack_expert_weights, pack_expert_weights_fp8
    g = torch.Generator(device="cuda").manual_seed(seed)
    tdt = torch.float32 if dtype == "f32" else torch.bfloat16

    def randn(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)
    gu = [randn(E + S, 2 * F, H, scale=H ** -0.5, dtype=tdt) for _ in range(L)]
    dn = [randn(E + S, H, F, scale=F ** -0.5, dtype=tdt) for _ in range(L)]
    desc = B.make_desc(L, H, F, E, k, S, D, dtype)
    if dtype == "fp8":
        W_gu, W_dn = pack_expert_weights_fp8(desc, gu, dn)
    else:
        W_gu, W_dn = [w.clone() for w in gu], [w.clone() for w in dn]
        pack_expert_weights(desc, W_gu, W_dn)
    G = next(n for n in (8, 4, 2) if E % n == 0)
    kw = dict(score="sigmoid", n_group=G, topk_group=G // 2, group_top=2 if E // G > 1 else 1, scale=2.5) if router else None
    x0 = randn(N, T, H)
    bal = randn(L, E, scale=0.1) if router and balance else None
    st = Stack(L=L, H=H, F=F, E=E, k=k, S=S, D=D, N=N, T=T, dtype=dtype, x=x0.clone(), gain=1 + randn(L, H, scale=0.1),
               Wg=[randn(E, H, scale=H ** -0.5, dtype=tdt) for _ in range(L)], bias=randn(L, E, scale=0.5), W_gu=W_gu,
               W_dn=W_dn, norm_topk=1, router=B.make_router(**kw) if router else None, balance=bal)
    return st, x0, (gu, dn), kw


STACKS = {
    "fp8_groups": dict(dtype="fp8", H=512, F=384, E=16, k=4, S=1, L=3, N=4, T=70),
    "fp8_plain": dict(dtype="fp8", H=512, F=256, E=8, k=2, S=0, L=2, N=3, T=40, router=False),
    "fp8_long_k": dict(dtype="fp8", H=256, F=8320, E=4, k=2, S=1, L=2, N=2, T=50),
    "fp8_decode": dict(dtype="fp8", H=1024, F=1024, E=32, k=4, S=1, L=2, N=4, T=6, balance=False),
    "bf16_groups": dict(dtype="bf16", H=512, F=384, E=64, k=6, S=2, L=2, N=4, T=50),
    "bf16_many": dict(dtype="bf16", H=512, F=128, E=256, k=8, S=1, L=2, N=3, T=33),
    "f32_groups": dict(dtype="f32", H=256, F=256, E=16, k=3, S=1, L=3, N=3, T=40),
}


@pytest.mark.parametrize("name", STACKS)
def test_every_driver_and_policy_gives_the_same_bits(name):
    st, x0, _, _ = make(seed=3, **STACKS[name])
    ref = None
    for policy, m in (("maxutil", 2), ("cumutil", 2), ("lockstep", None)):
        st.x.copy_(x0)
        steps = st.run(policy, m=m)
        torch.cuda.synchronize()
        loads = st.layer_loads.copy()
        if ref is None:
            ref = st.x.clone()
            assert torch.isfinite(ref).all() and not torch.equal(ref, x0)
        assert torch.equal(st.x, ref), (policy, "python")
        for dev in (False, True):
            st.x.copy_(x0)
            nat = st.run_native(policy, m=m, device_schedule=dev)
            torch.cuda.synchronize()
            assert torch.equal(st.x, ref), (policy, dev)
            assert np.array_equal(st.layer_loads, loads)
            assert [s.runset for s in nat] == [s.runset for s in steps]
            assert [s.groups for s in nat] == [s.groups for s in steps]


@pytest.mark.parametrize("name", ["fp8_groups", "fp8_decode", "fp8_plain"])
def test_each_stage_of_a_pass_against_the_oracle(name):
    st, x0, (gu, dn), kw = make(seed=4, **STACKS[name])
    L, H, F, E, k, S, N, T = st.L, st.H, st.F, st.E, st.k, st.S, st.N, st.T
    ES, slots, P = E + S, k + S, N * T * (k + S)
    c = Case.__new__(Case)
    c.P, c.F = P, F
    quant = [[o8.quantize_blocks(to64(w)) for w in layer] for layer in gu], [[o8.quantize_blocks(to64(w)) for w in layer] for layer in dn]
    c.gu, c.dn = ([(np.stack([q for q, _ in layer]), np.stack([s for _, s in layer])) for layer in part] for part in quant)
    c.h = torch.zeros(P * F + 4 * ((F + 511) // 512) * P, dtype=torch.uint8, device="cuda")
    before = {}

    def hook(stage, runset):
        torch.cuda.synchronize()
        assert [j for j, _ in runset] == list(range(N)) and len({l for _, l in runset}) == 1
        l = runset[0][1]
        if stage == "pre":
            before["x"] = st.x.clone()
            z = st.logits.cpu().numpy().reshape(-1, E)
            want = kw or dict(score="softmax", norm_topk=1)
            idx, w, _ = o8.select(z, k, balance=None if st.balance is None else st.balance[l].cpu().numpy(), **want)
            assert np.array_equal(st.idx.cpu().numpy().reshape(-1, k), idx)
            assert np.allclose(st.w.cpu().numpy().reshape(-1, k), w, rtol=2.0 ** -16, atol=0)
            for j in range(N):
                assert np.array_equal(st.counts[j].cpu().numpy(), np.bincount(idx[j * T:(j + 1) * T].reshape(-1), minlength=E))
            return
        idx = st.idx.cpu().numpy()
        perm, inv, off = operm.stable_permutation(operm.step_keys([(l, idx[j]) for j in range(N)], E, S), L * ES)
        assert np.array_equal(st.inv[:P].cpu().numpy(), inv)
        a, o, (hq, hs) = to64(st.a).reshape(N * T, H), to64(st.o[:P]), c.hidden()
        for key in np.nonzero(np.diff(off))[0]:
            rows = slice(off[key], off[key + 1])
            c.check_rows(rows, a[perm[rows] // slots], *divmod(int(key), ES), o, hq, hs)
        # the weighted sum: slots + 2 roundings of fp32
        w = np.concatenate([to64(st.w).reshape(N * T, k), np.ones((N * T, S))], axis=1)[:, :, None]
        rows = o[inv].reshape(N * T, slots, H)
        x = to64(before["x"]).reshape(N * T, H)
        size = np.abs(x) + (np.abs(w) * np.abs(rows)).sum(axis=1)
        assert (np.abs(to64(st.x).reshape(N * T, H) - (x + (w * rows).sum(axis=1))) <= (slots + 2) * o8.U * size).all()

    st.run("lockstep", views=dict(h=c.h), hook=hook)


def test_quantised_layers_and_a_checkpoint_pair_pack_alike():
    from paper_2608_07964_amd import binding as B
    from paper_2608_07964_amd.driver import is_packed, pack_expert_weights_fp8
    d = B.make_desc(1, 256, 128, 3, 1, 0, 1, "fp8")
    g = torch.Generator(device="cuda").manual_seed(1)
    gu, dn = (torch.randn(3, n, k, generator=g, device="cuda").to(torch.bfloat16) for n, k in ((256, 256), (256, 128)))
    pairs = []
    for w in (gu, dn):
        qs = [o8.quantize_blocks(to64(m)) for m in w]
        pairs.append((torch.from_numpy(np.stack([q for q, _ in qs]).astype(np.float32)).cuda().to(F8),
                      torch.from_numpy(np.stack([s for _, s in qs]).astype(np.float32)).cuda()))
    one, two = pack_expert_weights_fp8(d, [gu], [dn]), pack_expert_weights_fp8(d, [pairs[0]], [pairs[1]])
    for a, b in zip(one, two):
        assert torch.equal(a[0], b[0]) and is_packed(a[0])
    for bad in (gu[:2], gu.half(), (pairs[0][0], pairs[0][1][:, :1]), gu.transpose(1, 2)):
        with pytest.raises(ValueError):
            pack_expert_weights_fp8(d, [bad], [dn])
