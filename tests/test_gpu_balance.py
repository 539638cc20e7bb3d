"""The router's balance and z losses with per-expert counts and the gradient of the
logits (balance_loss) against the formulas in 64 bits; the gradient also against
differences; refusals.

Tolerances: counts are whole numbers and equal. exp and log of fp32 arguments up
to 90 in size are within (90 + 4) 2^-24 ~ 6e-6 of their values, a sum over 512
experts adds 21 roundings (1e-6), sums over tokens add at most 60 terms in a row
and a tree (5e-6): 2e-5 of the sum of the absolute values of the terms."""
import ctypes as C

import pytest
import torch


def reference(z, q, k, mask, wb, wz):
    """Losses, counts, mean probabilities and gradient in 64 bits, and the size of
    the gradient's terms."""
    z = z.double().cpu()
    T, K = z.shape
    valid = torch.ones(T, dtype=torch.bool) if mask is None else mask.cpu() != 0
    valid &= ~(z == float("-inf")).all(1)
    q, k = q.cpu().long(), torch.full((T,), q.shape[1]) if k is None else k.cpu()
    counts = torch.zeros(K, dtype=torch.int64)
    for t in torch.nonzero(valid)[:, 0].tolist():
        for j in q[t, :max(0, int(k[t]))].tolist():
            if 0 <= j < K:
                counts[j] += 1
    n = max(1, int(valid.sum()))
    f = counts.double() / max(1, int(counts.sum()))
    zv = z[valid]
    p, lse = torch.softmax(zv, 1), torch.logsumexp(zv, 1)
    P = p.sum(0) / n
    b, zl = K * (f * P).sum(), lse.square().sum() / n
    fp = (p * f).sum(1, keepdim=True)
    d, size = torch.zeros(T, K, dtype=torch.float64), torch.zeros(T, K, dtype=torch.float64)
    d[valid] = p / n * (wb * K * (f - fp) + 2 * wz * lse[:, None])
    size[valid] = p / n * (abs(wb) * K * (f + fp) + 2 * abs(wz) * (lse.abs() + 1)[:, None])
    return torch.stack([wb * b + wz * zl, b, zl]), counts, P, d, size


def check(z, q, k, mask, wb=0.02, wz=0.003):
    from paper_2608_10392_gb300 import balance_loss
    r = balance_loss(z, q, k, mask=mask, balance_weight=wb, z_weight=wz)
    loss, counts, P, d, size = reference(z, q, k, mask, wb, wz)
    assert torch.equal(r["counts"].cpu().long(), counts)
    assert ((r["prob"].double().cpu() - P).abs() <= 2e-5 * P + 1e-30).all()
    scale = torch.stack([abs(wb) * loss[1] + abs(wz) * loss[2], loss[1], loss[2] + 1])
    assert ((r["loss"].double().cpu() - loss).abs() <= 2e-5 * scale).all(), (r["loss"], loss)
    bad = (r["dlogits"].double().cpu() - d).abs() > 2e-5 * size + 1e-30
    assert not bad.any(), int(bad.sum())
    assert r["dlogits"].shape == z.shape
    return r


def make(T, K, dtype, seed=0, n_q=None, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(T, K, generator=g) * spread).to(dtype)
    q = torch.sort(z.float(), dim=1, descending=True, stable=True)[1].to(torch.int32)
    if n_q is not None:
        q = q[:, :n_q].contiguous()
    k = torch.randint(0, q.shape[1] + 1, (T,), generator=g, dtype=torch.int32)
    mask = (torch.rand(T, generator=g) < 0.7).to(torch.uint8)
    return z.cuda(), q.cuda(), k.cuda(), mask.cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(1, 1), (1, 4), (3, 5), (256, 4), (257, 8), (1000, 9), (77, 16),
                                 (4099, 32), (300, 33), (129, 64), (500, 100), (65, 128), (40, 200),
                                 (31, 512), (20000, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_against_64_bits(T, K, dtype):
    z, q, k, mask = make(T, K, dtype, seed=T + K, n_q=min(K, 6))
    check(z, q, None, None)
    z[mask == 0] = float("nan")  # padding is not read
    r = check(z, q, k, mask, wb=-0.5)
    assert not r["dlogits"][mask == 0].any()


@pytest.mark.gpu
def test_columns_of_the_router_product():
    """The residual experts' columns of [T][K + 1], as bf16 rows of odd stride, and
    selections as columns of a wider table."""
    z, q, k, mask = make(700, 8, torch.bfloat16, seed=1)
    wide = torch.cat([z[:, :1], z], 1)
    table = torch.cat([q, q], 1)
    check(wide[:, 1:], table[:, :8], k, mask)


@pytest.mark.gpu
def test_masked_logits_and_odd_selections():
    """Logits of -inf and of the type's lowest value, tokens without any expert left,
    selections out of range, repeated or negative in number."""
    z, q, k, _ = make(400, 12, torch.float32, seed=2)
    z[::3, 5] = float("-inf")
    z[1::3, 2] = torch.finfo(torch.float32).min
    z[7] = float("-inf")
    z[8] = torch.finfo(torch.float32).min
    q[11, 0], q[12, 0], q[13] = -1, 12, 3
    k[14], k[15] = -5, 100
    from paper_2608_10392_gb300 import balance_loss
    assert torch.isfinite(balance_loss(z, q, k)["dlogits"]).all()
    k[15] = 12
    z[8] = 0.5  # its logsumexp squared is beyond fp32; the rest has values to compare
    r = check(z, q, k, None)
    assert not r["dlogits"][7].any() and not r["dlogits"][::3, 5].any()


@pytest.mark.gpu
def test_large_logits():
    z, q, k, mask = make(300, 16, torch.float32, seed=3, spread=20.0)
    check(z + 1000.0, q, k, mask)


@pytest.mark.gpu
def test_nothing_to_do():
    """No token, only padding, or no selection: zeros, and no division by zero."""
    from paper_2608_10392_gb300 import balance_loss
    z, q, k, mask = make(50, 8, torch.float32)
    r = balance_loss(z[:0], q[:0], k[:0], z_weight=1.0)
    assert not r["loss"].any() and not r["counts"].any() and not r["prob"].any()
    r = balance_loss(z, q, k, mask=torch.zeros_like(mask), z_weight=1.0)
    assert not r["loss"].any() and not r["counts"].any() and not r["dlogits"].any()
    check(z, q, torch.zeros_like(k), mask)
    r = balance_loss(z, q, k, mask=mask, grad=False)
    assert r["dlogits"] is None


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the 64-bit loss, h = 1e-5: off by h^2 of third
    derivatives, far below the 2e-5 of the fp32 gradient's terms."""
    from paper_2608_10392_gb300 import balance_loss
    z, q, k, mask = make(60, 10, torch.float32, seed=4)
    r = balance_loss(z, q, k, mask=mask, balance_weight=0.7, z_weight=0.2)
    zc = z.double().cpu()
    g = torch.Generator().manual_seed(5)
    for _ in range(3):
        t, h = torch.randn(zc.shape, generator=g, dtype=torch.float64), 1e-5
        up, down = (reference(zc + s * h * t, q, k, mask, 0.7, 0.2)[0][0] for s in (1, -1))
        terms = r["dlogits"].double().cpu() * t
        assert abs(float(terms.sum() - (up - down) / (2 * h))) <= 2e-5 * float(terms.abs().sum()) + 1e-9


@pytest.mark.gpu
def test_repeatable_and_on_another_stream():
    from paper_2608_10392_gb300 import balance_loss
    z, q, k, mask = make(30000, 32, torch.bfloat16, seed=6)
    a = balance_loss(z, q, k, mask=mask, z_weight=0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = balance_loss(z, q, k, mask=mask, z_weight=0.1)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.gpu
def test_counts_follow_the_layers_routing():
    """q and the residual counts of a layer's own forward."""
    import workloads
    from gpu_helpers import run_gpu
    from paper_2608_10392_gb300 import balance_loss
    wl = workloads.make_workload(workloads.spec("tiny_f32"))
    g = run_gpu(wl)
    z = torch.from_numpy(g.p).cuda().float().log()  # by rank; any logits will do for the counts
    r = balance_loss(z, torch.from_numpy(g.q).cuda().int(), torch.from_numpy(g.k).cuda().int())
    want = [int(sum((int(m) >> j) & 1 for m in g.em)) for j in range(wl.spec.n_experts)]
    assert r["counts"].tolist() == want


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4096, 1 << 22], ids=["one_kernel", "two_kernels"])
def test_selections_beyond_32_bits(T):
    """2^31 selections in all (8.6 GB of them): their total does not fit in 32 bits. The
    same for 2^31 of one expert, whose count is then given as 2^31 - 1."""
    from paper_2608_10392_gb300 import balance_loss
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    K, n_q = 8, (1 << 31) // T
    pattern = torch.tensor([0, 0, 0, 1, 1, 2, 3, 4, 5, 6, 7, 7, 7, 7, 7, 7], dtype=torch.int32,
                           device="cuda")
    q = torch.empty(1 << 31, dtype=torch.int32, device="cuda")
    q.view(-1, 16).copy_(pattern.expand(1 << 27, 16))
    z = torch.randn(T, K, generator=torch.Generator("cuda").manual_seed(T), device="cuda")
    wb, wz = 0.02, 0.003
    p, lse = torch.softmax(z.double(), 1), torch.logsumexp(z.double(), 1)
    P, zl = p.mean(0), lse.square().mean()
    for counts in (torch.bincount(pattern.long(), minlength=K) << 27,
                   torch.tensor([0, 0, 0, 1 << 31, 0, 0, 0, 0], device="cuda")):
        if counts[3] == 1 << 31:
            q.fill_(3)
        r = balance_loss(z, q.view(T, n_q), balance_weight=wb, z_weight=wz)
        f = counts.double() / 2.0 ** 31
        b, fp = K * (f * P).sum(), (p * f).sum(1, keepdim=True)
        assert torch.equal(r["counts"].long(), counts.clamp(max=(1 << 31) - 1))
        want = torch.stack([wb * b + wz * zl, b, zl])
        assert ((r["loss"].double() - want).abs() <= 2e-5 * (want + 1)).all(), (r["loss"], want)
        d = p / T * (wb * K * (f - fp) + 2 * wz * lse[:, None])
        size = p / T * (wb * K * (f + fp) + 2 * wz * (lse.abs() + 1)[:, None])
        assert ((r["dlogits"].double() - d).abs() <= 2e-5 * size).all()


def test_more_selections_than_a_cta_counts_are_refused():
    """2^31 selections in a CTA's tokens, whose counts are 32-bit (no GPU needed)."""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    L = pkg.lib()
    p, n_q = C.c_void_p(4096), 1 << 30
    assert L.unif_moe_balance_loss(4, 8, p, 0, 8, p, n_q, n_q, None, None, 0.1, 0.1, p, p, p, None,
                                   None, 0, None) == -2
    assert b"selections" in L.unif_moe_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(40001, 3), (9001, 12), (3001, 50), (2100, 100), (700, 200), (333, 400)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_more_tokens_than_a_cluster_holds(T, K, dtype):
    """Two kernels, in each of their forms; also without a gradient, where the losses are
    the same."""
    from paper_2608_10392_gb300 import balance_loss
    z, q, k, mask = make(T, K, dtype, seed=T + K, n_q=min(K, 6))
    z[mask == 0] = float("nan")
    r = check(z, q, k, mask)
    assert torch.isfinite(r["dlogits"]).all()
    s = balance_loss(z, q, k, mask=mask, balance_weight=0.02, z_weight=0.003, grad=False)
    assert s["dlogits"] is None and all(torch.equal(r[n], s[n]) for n in ("loss", "counts", "prob"))


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(1, 4), (300, 33), (4099, 32), (31, 512)])
def test_losses_without_a_gradient(T, K):
    from paper_2608_10392_gb300 import balance_loss
    z, q, k, mask = make(T, K, torch.float32, seed=T, n_q=min(K, 6))
    s = balance_loss(z, q, k, mask=mask, balance_weight=0.02, z_weight=0.003, grad=False)
    loss, counts, P, _, _ = reference(z, q, k, mask, 0.02, 0.003)
    assert torch.equal(s["counts"].cpu().long(), counts)
    assert ((s["prob"].double().cpu() - P).abs() <= 2e-5 * P + 1e-30).all()
    assert ((s["loss"].double().cpu() - loss).abs() <= 2e-5 * (loss.abs() + 1)).all()


def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    L = pkg.lib()
    p = C.c_void_p(4096)

    def call(**k):
        a = dict(T=4, K=8, z=p, dtype=0, ld=8, q=p, n_q=2, ld_q=2, wb=0.1, wz=0.1, loss=p, counts=p,
                 prob=p)
        a.update(k)
        return L.unif_moe_balance_loss(a["T"], a["K"], a["z"], a["dtype"], a["ld"], a["q"], a["n_q"],
                                       a["ld_q"], None, None, a["wb"], a["wz"], a["loss"],
                                       a["counts"], a["prob"], None, None, 0, None)

    for k in (dict(T=-1), dict(K=0), dict(z=None), dict(dtype=2), dict(ld=7), dict(q=None),
              dict(n_q=-1), dict(ld_q=1), dict(wb=float("nan")), dict(wz=float("inf")),
              dict(loss=None), dict(counts=None), dict(prob=None)):
        assert call(**k) == -1, k
    assert call(K=513, ld=513) == -2
    assert L.unif_moe_balance_workspace(4, 0) == -1
    with pytest.raises(ValueError, match="logits"):
        pkg.balance_loss(torch.zeros(4, 8, dtype=torch.float16), torch.zeros(4, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="logits"):
        pkg.balance_loss(torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32))  # not on the GPU
