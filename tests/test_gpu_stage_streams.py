"""A stage on a stream of its own whose variant is set while the caller's stream is still busy with memory that it has
freed already: the variant's workspace is no part of it, and the results are those of a stage on the caller's stream."""
import pytest

import datagen
from gpu_common import log, shape_of, to_device
from test_gpu_stage_variant import F32, F64, _documents, _slopes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", [F32, F64], ids=lambda w: w.name)
def test_variant_on_a_stream_of_its_own(w):
    import torch
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd.stage import Stage
    log(w.name)
    dev = torch.device("cuda:0")
    dt = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    inp = to_device(datagen.step_inputs(w, 0), w, dev)
    ids, flags = (torch.from_numpy(t).to(dev) for t in _documents(w))
    slopes = torch.from_numpy(_slopes(w)).to(dev)
    names = list(datagen.init_params(w))
    results = []
    for stream in (None, torch.cuda.Stream(dev)):
        st = Stage(shape_of(w), "cuda:0", stream=stream)
        st.load_master(datagen.init_params(w))
        y, dx = (torch.full((w.micro_batch, w.seq_len, w.d_model), float("nan"), dtype=dt, device=dev) for _ in range(2))
        torch.cuda.synchronize()
        B.stage_sync_weights(st.handle)  # the master weights were written on the caller's stream
        torch.cuda.synchronize()
        held = []
        if stream is not None:  # blocks of every size that the workspace could take, freed with work on them to come
            held = [torch.empty(1 << s, dtype=torch.uint8, device=dev) for s in range(16, 27) for _ in range(2)]
            torch.cuda._sleep(200_000_000)
            spans = [(t.data_ptr(), t.data_ptr() + t.numel()) for t in held]
            for t in held:
                t.fill_(0x7F)
            del t
            held.clear()
        st.set_variant(softcap=2.0, dropout=0.25, seed=7, documents=True)
        if stream is not None:
            ws = st._variant[0]
            assert not any(lo < ws.data_ptr() + ws.numel() and ws.data_ptr() < hi for lo, hi in spans)
        st.set_documents(0, ids, flags)
        st.forward(0, 0, x_in=inp["x_in"], y_out=y)
        st.backward(0, dy=inp["dy"], dx_out=dx)
        torch.cuda.synchronize()
        first = [y.clone(), dx.clone(), *(st.view(f"grad0.{n}").clone() for n in names)]
        st.set_variant(softcap=2.0, slopes=slopes.clone(), documents=True)  # written by the caller's stream just now
        st.set_documents(0, ids, flags)
        st.forward(0, 0, x_in=inp["x_in"], y_out=y)
        st.backward(0, dy=inp["dy"], dx_out=dx)
        torch.cuda.synchronize()
        results.append([*first, y, dx])
        st.close()
    assert all(bool(torch.isfinite(t.float()).all()) for t in results[0])
    for a, b in zip(*results):
        assert torch.equal(a, b)
