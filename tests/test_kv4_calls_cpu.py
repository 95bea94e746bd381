"""What the Python calls of the 4-bit cache hand to the library, without a GPU:
host arrays have the lengths that it reads, tensors the types, sizes and device
that its kernels use.  The pool and the library are stand-ins."""

import contextlib
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from paper_2512_04752_amd import binding as B

CFG = wl.TINY


@pytest.fixture
def calls(monkeypatch):
    """The library's calls that get through."""
    got = []
    fake = SimpleNamespace(spec_verify_kv4=lambda *a: got.append("verify") or 0,
                           spec_kv4_commit=lambda *a: got.append("commit") or 0)
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(B, "_on", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(B, "_stream", lambda stream: None)
    return got


def pool():
    return SimpleNamespace(handle=None, cfg=CFG, index=0, buf=torch.empty(1, dtype=torch.uint8))


def verify(**changed):
    i32 = dict(dtype=torch.int32)
    a = dict(sample_ids=[0, 1], tree_offsets=[0, 3, 4], tree_tokens=[5, 6, 7, 8], tree_parents=[-1, 0, 0, -1],
             seq_lens=[10, 20], workspace=torch.empty(4096, dtype=torch.uint8), accepted_len=torch.empty(2, **i32),
             next_token=torch.empty(2, **i32), accepted_nodes=torch.empty(2, B.SPEC_MAX_TREE, **i32),
             temperature=0.7, draft_probs=torch.empty(4, CFG.vocab), uniforms=torch.empty(4, 2),
             debug=dict(logits=torch.empty(4, CFG.vocab), argmax=torch.empty(4, **i32), depth=None,
                        anc=torch.empty(4, B.SPEC_ANC_WORDS, dtype=torch.int64)))
    a.update(changed)
    weights = SimpleNamespace(struct=B.spec_weights())
    sv.spec_verify_kv4(CFG, weights, pool(), **a)


def commit(**changed):
    a = dict(sample_ids=[0, 1], seq_lens=[10, 20], accepted_len=torch.empty(2, dtype=torch.int32),
             accepted_nodes=torch.empty(2, B.SPEC_MAX_TREE, dtype=torch.int32),
             new_seq_lens=torch.empty(2, dtype=torch.int32))
    a.update(changed)
    sv.spec_kv4_commit(pool(), **a)


def test_calls_that_are_in_order(calls):
    verify()
    verify(temperature=0.0, draft_probs=None, uniforms=None, debug=None)
    commit()
    assert calls == ["verify", "verify", "commit"]


ELSEWHERE = torch.empty(1 << 16, dtype=torch.uint8, device="meta")      # not the pool's device


@pytest.mark.parametrize("changed", [
    dict(seq_lens=[10]), dict(seq_lens=[10, 20, 30]), dict(tree_offsets=[0, 4]), dict(tree_offsets=[0, 3, 4, 5]),
    dict(tree_tokens=[5, 6, 7]), dict(tree_parents=[-1, 0, 0]), dict(tree_offsets=[0, 3, 400]),
    dict(sample_ids=[0]),
    dict(workspace=ELSEWHERE), dict(workspace=torch.empty(4096, dtype=torch.int32)),
    dict(workspace=torch.empty(64, 64, dtype=torch.uint8)[:, ::2]),
    dict(draft_probs=torch.empty(4, CFG.vocab, device="meta")), dict(uniforms=torch.empty(4, 2, device="meta")),
    dict(draft_probs=torch.empty(3, CFG.vocab)), dict(uniforms=None),
    dict(accepted_len=torch.empty(1, dtype=torch.int32)), dict(next_token=torch.empty(2, dtype=torch.int64)),
    dict(accepted_nodes=torch.empty(2, 8, dtype=torch.int32)),
    dict(debug=dict(logits=torch.empty(3, CFG.vocab))), dict(debug=dict(argmax=torch.empty(4, dtype=torch.int64))),
    dict(debug=dict(pos=torch.empty(4, dtype=torch.int32, device="meta"))),
    dict(debug=dict(anc=torch.empty(4, dtype=torch.int64))),
], ids=lambda c: "-".join(c))
def test_verify_refusals(calls, changed):
    with pytest.raises(ValueError):
        verify(**changed)
    assert not calls


@pytest.mark.parametrize("changed", [
    dict(seq_lens=[10]), dict(seq_lens=[10, 20, 30]), dict(sample_ids=[0, 1, 2]), dict(seq_lens=np.empty(0, np.int32)),
    dict(accepted_len=torch.empty(2, dtype=torch.int32, device="meta")),
    dict(new_seq_lens=torch.empty(1, dtype=torch.int32)),
], ids=lambda c: "-".join(c))
def test_commit_refusals(calls, changed):
    with pytest.raises(ValueError):
        commit(**changed)
    assert not calls


@pytest.mark.parametrize("offsets,parents,lens", [([0, 1], [-1], [5, 6]), ([0], None, []), ([0, 3], [-1, 0], [5])])
def test_step_refusals(offsets, parents, lens):
    with pytest.raises(ValueError):
        sv.KV4Step(pool(), [0], offsets, parents, lens, workspace=torch.empty(64, dtype=torch.uint8))


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu")], ids=str)
def test_pool_off_the_device(device):
    with pytest.raises(ValueError, match="device memory"):
        sv.KV4Pool(CFG, 1, 2, device=device)
    with pytest.raises(ValueError):
        sv.KV4Pool(CFG, 1, 2, buf=torch.empty(1 << 20, dtype=torch.uint8))


def test_streams_of_another_device(calls):
    """Launched there, the kernels would take the pool's addresses for their own device's."""
    here, there = (SimpleNamespace(cuda_stream=7, device=torch.device("cuda", i)) for i in (0, 1))
    for call in (verify, commit):
        with pytest.raises(ValueError, match="stream"):
            call(stream=there)
        call(stream=here)
    assert calls == ["verify", "commit"]
    with pytest.raises(ValueError, match="stream"):
        sv.KV4Step(pool(), [0], [0, 1], None, [5], stream=there)
    step = sv.KV4Step.__new__(sv.KV4Step)
    step.handle, step.pool, step._made_on = None, pool(), None
    step.pool.handle = 1
    assert step._on_stream(here) == 7
    with pytest.raises(ValueError, match="stream"):
        step._on_stream(there)
