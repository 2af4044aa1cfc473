"""A wait that runs out in a context whose memory held other things before.

A forward whose wait gave up leaves its greedy choices unwritten, and launches are queued behind it that take them for tokens.  The context's memory
comes from the caller and may hold anything: whatever it held, the call has to end with OURO_ETIMEOUT, and the same context has to decode as one on
cleared memory does once it is given time again.
"""
import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import binding, synth

gpu = pytest.mark.gpu
WIDE = synth.ModelDesc(3, 256, 8, 2, 64, 512, 1000, 320, "bf16")      # split tiles of the tensor cores
NARROW = synth.ModelDesc(2, 64, 4, 2, 32, 96, 100, 192, "f32")        # one launch for the whole forward
PLAIN = synth.ModelDesc(2, 576, 8, 2, 64, 704, 500, 192, "f32")       # a launch for each step
P = synth.DecodeParams(4, 9, 4, 16, 8)


def engine(monkeypatch, desc, byte, draft=False):
    """An engine whose memory held `byte` everywhere when it was made."""
    w = synth.model_weights(desc, 2, device="cuda:0")

    def filled(*size, **kw):
        t = torch.zeros(*size, **kw)
        return t.fill_(byte) if t.dtype == torch.uint8 else t

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", filled)
        return binding.Engine(desc, w, P, desc if draft else None, w if draft else None)


@gpu
@pytest.mark.parametrize("byte", [0x5a, 0xff])
@pytest.mark.parametrize("desc", [WIDE, NARROW, PLAIN], ids=["wide", "narrow", "plain"])
def test_whatever_the_memory_held(monkeypatch, desc, byte):
    prompt = synth.prompt(2, desc.vocab, 40, 0.4, 4, 8)
    clear = engine(monkeypatch, desc, 0, draft=True)
    want, _ = clear.generate_vanilla(prompt, 12)
    spec, _ = clear.generate(prompt, 12)
    clear.close()
    eng = engine(monkeypatch, desc, byte, draft=True)
    try:
        if desc is not PLAIN:                              # has no waits, and refuses to limit them
            eng.set_wait_limit(0)
        for call, right in ((eng.generate_vanilla, want), (eng.generate, spec)):
            if desc is PLAIN:
                assert np.array_equal(call(prompt, 12)[0], right)
                continue
            with pytest.raises(binding.OuroError) as e:
                call(prompt, 12)
            assert e.value.status == binding.OURO_ETIMEOUT
        if desc is not PLAIN:
            eng.set_wait_limit(-1)
        assert np.array_equal(eng.generate_vanilla(prompt, 12)[0], want)
        assert np.array_equal(eng.generate(prompt, 12)[0], spec)
    finally:
        if desc is not PLAIN:
            eng.set_wait_limit(-1)
        eng.close()


@gpu
@pytest.mark.parametrize("desc", [WIDE, NARROW, PLAIN], ids=["wide", "narrow", "plain"])
def test_tokens_outside_the_table_read_some_row_of_it(monkeypatch, desc):
    """assemble_candidates and verify_forward take tokens from device memory, which nobody has checked."""
    eng = engine(monkeypatch, desc, 0)
    prompt = synth.prompt(2, desc.vocab, 40, 0.4, 4, 8)
    got = []
    for bad in (desc.vocab - 1, desc.vocab, 2 ** 31 - 1, -1):
        eng.reset()
        eng.prefill(prompt[:20])
        eng.assemble_candidates(draft=[1, 2, 3, bad])
        eng.verify_forward()
        torch.cuda.synchronize()
        got.append(eng.argmax[:5].tolist())
    eng.close()
    assert all(g[:4] == got[0][:4] for g in got)
    assert all(0 <= t < desc.vocab for g in got for t in g)
