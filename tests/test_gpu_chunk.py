"""Steps that bring chunks of prompts, all operators together as a server uses
them: tables built on the GPU, slice blocks with older tokens prefetched, the
chunk's K and V stored, causal attention, the touched staged copies written back --
chunk after chunk until the prompts are in, then a decode step on the path that was
there before, and differential attention over the same cache. An oracle replays the
block movement; attention is compared every layer and step, both pools byte for
byte."""
import numpy as np
import pytest
import torch

import oracle
import synth
from harness import TORCH_DT, Workload, oracle_mirror, rel_err
from ops_harness import assert_close, dev16
from oracle import ops as oops
from paper_2609_27040_amd.step import run_chunk

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def replay(st, w, l, chunk, k, v):
    """The oracle's prefetch, store and write-back of a layer; its attention table."""
    ids = [w.tables[l][w.tables[l] >= 0]]
    ref = oops.kv_tables(ids, w.lens, chunk.new, w.maxblk, w.bs, w.n_local, chunk.T,
                         w.staging[l % w.staging_slots][None], 10 ** 4)
    n = int(ref["prefetch"][2][0])
    st.prefetch(ref["prefetch"][0][0, :n], ref["prefetch"][1][0, :n])
    oops.kv_store(st.local, k, v, ref["slots"][0], w.hkv, w.D, w.bs)
    m = int(ref["writeback"][2][0])
    assert (n, m) == (chunk.n_prefetch[l], chunk.n_writeback[l])
    st.writeback(ref["writeback"][0][0, :m], ref["writeback"][1][0, :m])
    return ref


def same_pools(w, st):
    torch.cuda.synchronize()
    assert np.array_equal(w.local_view.cpu().numpy(), st.local)
    assert np.array_equal(w.slice_view.cpu().numpy(), st.slice)


@pytest.mark.parametrize("layout,graph", [(0, False), (1, False), (0, True)])
def test_prompts_in_chunks_then_a_decode_step(layout, graph):
    cfg = synth.TINY.scaled(q_heads=8, kv_heads=2, dtype="bf16")
    full = np.array([130, 17, 64, 1, 200])
    w = Workload(cfg, layers=4, slice_layout=layout, staging_slots=2, lens=full, frac=0.4)
    st = oracle_mirror(w)
    rng = np.random.default_rng(5)
    dt = TORCH_DT["bf16"]
    try:
        done = np.zeros(len(full), np.int64)
        for take in (50, 77, 200):                     # ragged chunks; some sequences are done early
            new = np.minimum(full - done, take)
            done += new
            w.lens = done.copy()
            w.lens_dev.copy_(torch.from_numpy(done.astype(np.int32)))
            # blocks behind the tokens that are there yet are not part of the step
            keep = w.tables.copy()
            w.tables[:, np.arange(w.maxblk)[None, :] >= -(-done // w.bs)[:, None]] = -1
            chunk = w.chunk(new)
            T = chunk.T
            data = [[synth.random_16bit(rng, (T, h, w.D), "bf16") for h in (8, 2, 2)]
                    for _ in range(w.L)]
            dev = [[dev16(x, "bf16") for x in d] for d in data]
            outs = [torch.zeros((T, 8, w.D), dtype=dt, device="cuda") for _ in range(w.L)]
            layer = lambda l: (*dev[l], outs[l])
            if graph:
                s = torch.cuda.Stream()
                s.wait_stream(torch.cuda.current_stream())
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    run_chunk(w, chunk, layer, stream=s)
                before = [v.clone() for v in (w.local_view, w.slice_view)]
                for _ in range(3):                     # the same step from the same pools
                    w.local_view.copy_(before[0])
                    w.slice_view.copy_(before[1])
                    for o in outs:
                        o.zero_()
                    torch.cuda.synchronize()
                    g.replay()
                    torch.cuda.synchronize()
            else:
                run_chunk(w, chunk, layer)
            for l in range(w.L):
                q, k, v = data[l]
                ref = replay(st, w, l, chunk, k, v)
                assert np.array_equal(chunk.block_table[l].cpu().numpy(), ref["table"][0])
                assert np.array_equal(chunk.slots[l].cpu().numpy(), ref["slots"][0])
                want, mass = oops.prompt_attention(q, ref["starts"], ref["table"][0], w.lens,
                                                   st.read_block, 2, w.D, w.bs, "bf16")
                assert_close(outs[l], want, mass, dt, "bf16", int(w.lens.max()))
                # differential attention of the same chunk, over the same staged blocks:
                # the last layers' copies are still in place
                if l >= w.L - w.staging_slots and T:
                    lam = np.linspace(0.2, 0.9, 4).astype(np.float32)
                    got = torch.zeros((T, 4, 2 * w.D), dtype=torch.float32, device="cuda")
                    w.diff_prompt_attention(l, chunk, dev[l][0], torch.tensor(lam, device="cuda"),
                                            got)
                    want, mass = oops.prompt_attention(q, ref["starts"], ref["table"][0], w.lens,
                                                       st.read_block, 2, w.D, w.bs, "bf16", lam=lam)
                    assert_close(got, want, mass, torch.float32, "bf16", int(w.lens.max()))
            same_pools(w, st)
            w.tables = keep
        # the prompts are in: a decode step as before, and differential attention of its token
        w.restage()
        lam = np.array([0.5, 0.25, 0.7, 0.1], np.float32)
        for l in range(w.L):
            w.prefetch(l)
            st.prefetch(w.pf_src[l], w.pf_dst[l])
            out = w.new_out()
            w.attention(l, out)
            ref = oracle.paged_decode_attention(w.q16, w.attn_tables[l], w.lens, st.read_block, 2,
                                                w.D, w.bs, "bf16")
            assert rel_err(out.cpu().numpy(), ref) <= 2e-3
            diff = torch.zeros((w.B, 4, 2 * w.D), dtype=torch.float32, device="cuda")
            w.diff_attention(l, w.q, torch.tensor(lam, device="cuda"), diff)
            want, mass = oops.prompt_attention(w.q16, np.arange(w.B + 1), w.attn_tables[l], w.lens,
                                               st.read_block, 2, w.D, w.bs, "bf16", lam=lam)
            assert_close(diff, want, mass, torch.float32, "bf16", int(w.lens.max()))
        from paper_2609_27040_amd import ema
        assert ema.slice_device_errors(w.h) == 0
    finally:
        w.close()


def test_tables_built_on_another_stream():
    cfg = synth.TINY.scaled(q_heads=8, kv_heads=2, dtype="bf16")
    w = Workload(cfg, layers=3, slice_layout=0, staging_slots=2, lens=np.array([90, 33]), frac=0.5)
    try:
        here = w.chunk([40, 33])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        torch.cuda._sleep(20_000_000)
        there = w.chunk([40, 33], stream=side)
        torch.cuda.synchronize()
        for a, b in ((here.block_table, there.block_table), (here.slots, there.slots),
                     (here.starts, there.starts), *zip(here.prefetch, there.prefetch),
                     *zip(here.writeback, there.writeback)):
            assert torch.equal(a, b)
        for bad in ([40], [91, 1], [-1, 1]):
            with pytest.raises(ValueError):
                w.chunk(bad)
    finally:
        w.close()
