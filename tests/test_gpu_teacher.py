"""A teacher's top logits in the loss of the server step, against the oracle's round with the loss of its definition in 64 bits.
The rest of the step is the same arithmetic as without a teacher, so the tolerances are those of the other parity tests."""
import numpy as np
import pytest
import torch

import harness as H
from oracle import splitlora_oracle as O
from paper_2407_00952_b200 import binding as B
from paper_2407_00952_b200 import runner, synth

pytestmark = pytest.mark.gpu

TOL_FP32, TOL_BF16, TOL_LOSS = 1e-4, 2e-2, 1e-3


def make_teacher(w, k, seed=5):
    """top_idx, top_logits [K, b, T, k]: k different entries per position, some absent, some positions without any."""
    rng = np.random.default_rng(seed)
    shape = (w.n_clients, w.batch_per_client, w.seq)
    n = int(np.prod(shape))
    idx = np.stack([rng.permutation(w.vocab)[:k] for _ in range(n)]).reshape(shape + (k,)).astype(np.int32)
    t = (4 + 2 * rng.normal(size=shape + (k,))).astype(np.float32)
    idx[:, 0, ::5, k // 2:] = -1
    idx[0, -1, 3] = w.vocab + 7
    return idx, t


def distill64(z, labels, idx, t, T, wc, wk, V):
    """loss, dz from the definition, numpy."""
    idx, t = idx.reshape(len(z), -1), t.reshape(len(z), -1).astype(np.float64)
    take = (labels >= 0) & (labels < V)
    n = take.sum()
    dz, loss = np.zeros_like(z), 0.0

    def logsm(v):
        v = v - v.max()
        return v - np.log(np.exp(v).sum())

    for m in np.nonzero(take)[0]:
        ok = (idx[m] >= 0) & (idx[m] < V)
        if ok.any():
            lq, lp = logsm(t[m][ok] / T), logsm(z[m] / T)
            q = np.exp(lq)
            loss += wk * T * T * (q * (lq - lp[idx[m][ok]])).sum()
            g = np.exp(lp)
            np.subtract.at(g, idx[m][ok], q)
            dz[m] += wk * T * g
        lp = logsm(z[m])
        loss -= wc * lp[labels[m]]
        g = np.exp(lp)
        g[labels[m]] -= 1
        dz[m] += wc * g
    return float(loss / n), dz / n


def run(w, case, teacher=None, monkeypatch=None, T=2.0, wc=0.4, wk=0.6, calls=True):
    frozen, cads, sads, tokens, labels = case
    eng = runner.make_engine(w, frozen, cads, sads, optimizer="sgd")
    if teacher is not None:
        idx, t = teacher
        eng.set_teacher(torch.from_numpy(idx).cuda(), torch.from_numpy(t).cuda(), temperature=T, ce_weight=wc, kd_weight=wk)
    S, dS = eng.new_activation_buffer(), eng.new_activation_buffer()
    eng.client_fwd(torch.from_numpy(tokens).cuda(), S)
    loss = eng.server_step(S, torch.from_numpy(labels).cuda(), dS)
    eng.client_bwd(dS)
    torch.cuda.synchronize()
    assert eng.device_status() == 0
    return eng, S, dS, loss


def parity(w, monkeypatch, tol, T=2.0, k=12):
    case = H.build_case(w)
    case[4][0, 0, 3:9] = -1
    teacher = make_teacher(w, k)
    monkeypatch.setattr(O, "cross_entropy_fwd_bwd", lambda z, lab: distill64(z, lab, *teacher, T, 0.4, 0.6, w.vocab))
    eng, S, dS, loss = run(w, case, teacher, T=T)
    _, _, _, _, S_ref, dS_ref, loss_ref, sg, cg = H.oracle_three_calls(w, *case, optimizer="sgd")
    assert abs(loss - loss_ref) <= TOL_LOSS * abs(loss_ref)
    assert H.rel_err(H.tnp(dS), dS_ref) <= tol
    for (l, t), (dA, dB) in sg.items():
        gA, gB = eng.get_adapter_grad(B.SIDE_SERVER, 0, l, B.TARGET_BITS[t])
        assert H.rel_err(H.tnp(gA), dA) <= tol and H.rel_err(H.tnp(gB), dB) <= tol, ("server", l, t)
    for i in range(w.n_clients):
        for (l, t), (dA, dB) in cg[i].items():
            gA, gB = eng.get_adapter_grad(B.SIDE_CLIENT, i, l, B.TARGET_BITS[t])
            assert H.rel_err(H.tnp(gA), dA) <= tol and H.rel_err(H.tnp(gB), dB) <= tol, ("client", i, l, t)
    return eng


@pytest.mark.parametrize("T", [1.0, 2.0, 1.3])
def test_teacher_fp32_round(monkeypatch, T):
    parity(synth.WORKLOADS[1], monkeypatch, TOL_FP32, T=T)


def test_teacher_bf16_round(monkeypatch):
    """A vocabulary that is no multiple of the head's padded width: the padding columns stay zero in the gradient."""
    # adapters on v only: the looser bound of q and k gradients (harness.QK_BOUND) is not what is looked at here
    w = synth.scaled(synth.WORKLOADS[3], n_layer=2, cut=1, n_clients=2, batch_per_client=1, seq=256, max_seq=256, vocab=2050, targets=("v",))
    parity(w, monkeypatch, TOL_BF16)


def test_teacher_that_says_the_label_is_the_cross_entropy():
    """One entry, the label: q is one there, so at T = 1 the divergence is the cross-entropy, and so are all gradients."""
    w = synth.WORKLOADS[1]
    case = H.build_case(w)
    labels = case[4]
    one = (labels[..., None].astype(np.int32), np.zeros(labels.shape + (1,), np.float32))
    eng0, _, dS0, loss0 = run(w, case)
    eng1, _, dS1, loss1 = run(w, case, one, T=1.0, wc=0.0, wk=1.0)
    assert abs(loss1 - loss0) <= 1e-6 * abs(loss0)
    assert H.rel_err(H.tnp(dS1), H.tnp(dS0)) <= 1e-5
    # and without a teacher again
    eng1.set_teacher(None)
    S, dS = eng1.new_activation_buffer(), eng1.new_activation_buffer()
    eng1.client_fwd(torch.from_numpy(case[3]).cuda(), S)
    eng0.client_fwd(torch.from_numpy(case[3]).cuda(), S)
    assert abs(eng0.server_step(S, torch.from_numpy(labels).cuda(), dS) - eng1.server_step(S, torch.from_numpy(labels).cuda(), dS)) <= 1e-4


def test_teacher_in_whole_rounds_with_a_shard_normaliser():
    """round() takes the teacher too; a normaliser of twice the count halves the loss."""
    w = synth.WORKLOADS[1]
    frozen, cads, sads, tokens, labels = H.build_case(w)
    idx, t = make_teacher(w, 8)
    counts = synth.make_counts(w)
    losses = []
    for norm in (0, 2 * labels.size):
        eng = runner.make_engine(w, frozen, cads, sads, optimizer="adamw")
        eng.set_teacher(torch.from_numpy(idx).cuda(), torch.from_numpy(t).cuda(), temperature=2.0)
        eng.set_loss_normalizer(norm)
        losses.append(eng.round(torch.from_numpy(tokens).cuda(), torch.from_numpy(labels).cuda(), counts))
        eng.profile_enable(1)
        eng.round(torch.from_numpy(tokens).cuda(), torch.from_numpy(labels).cuda(), counts)
        rep = eng.profile_report()
        assert "distill_loss" in rep and "cross_entropy" not in rep
    assert abs(losses[0] - 2 * losses[1]) <= 1e-5 * losses[0]


def test_teacher_refusals():
    w = synth.WORKLOADS[1]
    frozen, cads, sads, tokens, labels = H.build_case(w)
    eng = runner.make_engine(w, frozen, cads, sads)
    idx, t = (torch.from_numpy(a).cuda() for a in make_teacher(w, 8))
    for args, kw in (((idx.long(), t), {}), ((idx, t.half()), {}), ((idx, None), {}), ((idx[:, :, :-1], t), {}), ((idx.cpu(), t.cpu()), {}),
                     ((idx, t), {"temperature": 0.0}), ((idx, t), {"temperature": float("nan")}), ((idx, t), {"ce_weight": float("inf")}),
                     ((torch.zeros(idx.shape[:-1] + (257,), dtype=torch.int32, device="cuda"), torch.zeros(idx.shape[:-1] + (257,), dtype=torch.float32, device="cuda")), {})):
        with pytest.raises(B.SplitLoraError) as e:
            eng.set_teacher(*args, **kw)
        assert e.value.code == -1
