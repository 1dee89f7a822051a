"""The operators at the two ends of a model as a program uses them: around the layer of a training iteration, and in a tied model
without a layer whose whole gradient is known."""
import numpy as np
import pytest

from paper_2510_03283_amd import synth
from test_gpu_parity import custom_workload

pytestmark = pytest.mark.gpu


def test_iteration_from_token_ids(torch_mod):
    """Embedding, layer, logits of the inference rows, their tokens' log-probabilities; then the DPO head, the layer's backward pass
    and the lookup's gradient on top of the head's: the whole gradient of the tied table."""
    torch = torch_mod
    from paper_2510_03283_amd import binding as B
    from paper_2510_03283_amd.harness import DeviceIteration
    dims = synth.ModelDims(512, 8, 2, 64, 1408, 8192, io_bf16=True)
    wl = custom_workload("ends", dims, prefill=(37, 130, 1), decode=(5, 300, 0, 77), n_pairs=2, prompt=20, resp=(9, 40))
    it = DeviceIteration(wl)
    try:
        ids = torch.from_numpy(wl.batch.token_ids.astype(np.int32)).cuda()
        want_x = it.x.clone()
        it.x.fill_(float("nan"))
        it.embed(ids)
        torch.cuda.synchronize()
        assert torch.equal(it.x, want_x)                       # the rows that the workload was made with
        it.step()
        n = it.Ti
        logits, tok = torch.empty((n, dims.vocab), device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        B.mace_next_token_logits(it.h, it.y, None, n, it.gf, it.E, logits, tok, it.ws)
        logp, top, top_logp = torch.empty(n, device="cuda"), torch.empty((n, 4), dtype=torch.int32, device="cuda"), torch.empty((n, 4), device="cuda")
        ws = torch.empty(B.mace_token_logprobs_workspace_bytes(it.h, n, dims.vocab, 4), dtype=torch.uint8, device="cuda")
        B.mace_token_logprobs(it.h, logits, ws, tok, logp, top_ids=top, top_logp=top_logp)
        head = it.dE.clone()
        it.embed_grad(ids[it.Ti:])
        torch.cuda.synchronize()
        assert torch.equal(top[:, 0], tok) and torch.equal(top_logp[:, 0], logp)      # the greedy token is the first alternative
        ref = torch.log_softmax(logits.double(), dim=1).gather(1, tok.long()[:, None])[:, 0]
        assert (logp.double() - ref).abs().max() <= 1e-5
        want = head.double().index_add_(0, ids[it.Ti:].long(), it.dx.double())
        assert (it.dE.double() - want).abs().max() <= 2.0 ** -24 * 200 * want.abs().max()     # at most 117 rows of one token and the head's
    finally:
        it.close()


def test_tied_model_learns_from_its_whole_gradient(torch_mod):
    """x = E[ids], logits = x E^T, loss = -sum logp - c sum H: forward and backward by the library alone, the table's gradient against
    the formula in 64 bits and against the change of the loss along a direction."""
    torch = torch_mod
    from paper_2510_03283_amd import binding as B
    d, V, n, c = 128, 640, 256, 0.25
    gen = torch.Generator(device="cuda").manual_seed(0)
    E = (0.2 * torch.randn((V, d), generator=gen, device="cuda")).to(torch.bfloat16)
    ids = torch.randint(0, V, (n,), generator=gen, device="cuda").int()
    label = torch.randint(0, V, (n,), generator=gen, device="cuda").int()
    label[5] = -1                                                            # padding
    h = B.mace_create(d, 2, 2, 64, 64, V, 1e-6, 1e4, B.MACE_BF16)
    try:
        f = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")
        x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
        logits, logp, ent, stats = f(n, V), f(n), f(n), f(n, 2)
        ws = torch.empty(max(B.mace_token_logprobs_workspace_bytes(h, n, V, 0), B.mace_embed_grad_workspace_bytes(h, n)), dtype=torch.uint8, device="cuda")
        B.mace_embed_tokens(h, E, ids, x)
        B.mace_gemm_bf16(h, 0, 0, n, V, d, x, E, logits)
        B.mace_token_logprobs(h, logits, ws, label, logp, ent, stats)
        dl = torch.empty((n, V), dtype=torch.bfloat16, device="cuda")
        B.mace_token_logprobs_grad(h, logits, stats, dl, label, torch.full((n,), -1.0, device="cuda"), ent, torch.full((n,), -c, device="cuda"))
        dx, dE = f(n, d), f(V, d)
        B.mace_gemm_bf16(h, 0, 1, n, d, V, dl, E, dx)
        B.mace_gemm_bf16(h, 1, 1, V, d, n, dl, x, dE)
        B.mace_embed_tokens_grad(h, ids, dx, dE, ws, accumulate=True)
        torch.cuda.synchronize()

        def loss(table):
            rows = table[ids.long()]
            lp = torch.log_softmax(rows @ table.T, dim=1)
            picked = lp.gather(1, label.clamp(min=0).long()[:, None])[:, 0][label >= 0]
            return -picked.sum() - c * torch.special.entr(lp.exp()).sum()

        table = E.double().cpu()
        ids, label = ids.cpu(), label.cpu()
        leaf = table.clone().requires_grad_()
        (want,) = torch.autograd.grad(loss(leaf), leaf)
        got = dE.double().cpu()
        # the one rounding to 8 bits is that of dl (half a step of 2^-8 each, 2^-8 / sqrt(3) of it in the mean square; the products then add with random signs)
        assert (got - want).norm() <= 2.0 ** -8 * want.norm()
        u = want / want.norm()
        slope = (loss(table + 1e-4 * u) - loss(table - 1e-4 * u)) / 2e-4
        assert abs((got * u).sum() - slope) <= 2.0 ** -8 * abs(slope)
    finally:
        B.mace_destroy(h)
