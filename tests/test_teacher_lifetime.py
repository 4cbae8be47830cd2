"""How long the memory of a teacher's logits lasts: until the steps that read it are done, whichever stream they run on."""
import types

import pytest
import torch

import harness as H
from paper_2407_00952_b200 import binding as B
from paper_2407_00952_b200 import runner, synth


class Stand:
    """Stands for a tensor on a device: what set_teacher looks at, and the streams it was recorded on."""
    is_cuda = True

    def __init__(self, dtype, shape, device):
        self.dtype, self.shape, self.device, self.recorded = dtype, torch.Size(shape), device, []

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, s):
        self.recorded.append(s)


def engine(accept):
    e = B.SplitLoRA.__new__(B.SplitLoRA)
    e.ctx, e.stream = None, object()
    e.cfg = types.SimpleNamespace(n_clients=2, batch_per_client=1, seq=4)
    e.workspace = types.SimpleNamespace(device="cuda:0")
    e.lib = types.SimpleNamespace(splitlora_set_teacher=lambda *a: 0 if accept else -1, splitlora_last_error=lambda c: b"refused")
    return e


def test_a_teacher_is_recorded_on_the_contexts_stream():
    e = engine(True)
    first, second = ([Stand(torch.int32, (2, 1, 4, 3), "cuda:0"), Stand(torch.float32, (2, 1, 4, 3), "cuda:0")] for _ in range(2))
    for pair in (first, second):
        e.set_teacher(*pair)
        assert all(t.recorded == [e.stream] for t in pair) and e.teacher == tuple(pair)
    e.set_teacher(None)
    assert e.teacher is None


def test_a_refused_teacher_leaves_the_last_one():
    e = engine(True)
    pair = [Stand(torch.int32, (2, 1, 4, 3), "cuda:0"), Stand(torch.float32, (2, 1, 4, 3), "cuda:0")]
    e.set_teacher(*pair)
    e.lib.splitlora_set_teacher = lambda *a: -1
    bad = [Stand(torch.int32, (2, 1, 4, 3), "cuda:0"), Stand(torch.float32, (2, 1, 4, 3), "cuda:0")]
    with pytest.raises(B.SplitLoraError):
        e.set_teacher(*bad, temperature=0.0)
    assert e.teacher == tuple(pair) and not bad[0].recorded


@pytest.mark.gpu
def test_a_teacher_replaced_while_its_step_is_under_way():
    w = synth.WORKLOADS[1]
    frozen, cads, sads, tokens, labels = H.build_case(w)
    shape = (w.n_clients, w.batch_per_client, w.seq, 16)
    g = torch.Generator(device="cuda").manual_seed(3)

    def teacher():
        return (torch.randint(0, w.vocab, shape, device="cuda", generator=g, dtype=torch.int32), 4 + 2 * torch.randn(shape, device="cuda", generator=g, dtype=torch.float32))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        eng = runner.make_engine(w, frozen, cads, sads, optimizer="sgd", lr_server=0.0)
    S, dS = eng.new_activation_buffer(), eng.new_activation_buffer()
    tok, lab = torch.from_numpy(tokens).cuda(), torch.from_numpy(labels).cuda()
    idx, t = teacher()
    torch.cuda.synchronize()
    eng.client_fwd(tok, S)
    eng.set_teacher(idx, t, temperature=2.0)
    want = eng.server_step(S, lab, dS)
    grad = dS.clone()
    others = [torch.full(shape, float("nan"), device="cuda") for _ in range(8)]           # the allocator's room, and the kernel's loading
    del others
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)           # half a second in front of the step
    eng.server_step(S, lab, dS, want_loss=False)
    eng.set_teacher(None)
    places = {idx.data_ptr(), t.data_ptr()}
    del idx, t
    others = [torch.full(shape, float("nan"), device="cuda") for _ in range(8)]           # on the current stream, which does not wait
    assert not side.query(), "the step was over too early for this test"
    assert not places & {o.data_ptr() for o in others}
    torch.cuda.synchronize()
    assert float(eng.loss_tensor()) == want and torch.equal(dS, grad)
