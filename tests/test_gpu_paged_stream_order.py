"""The paged beam search's operators in a stream: their kernels may be placed before the one ahead of them has ended,
and still see all that it wrote.  The same calls with a synchronisation after each give the same bits."""
import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu

HEADS, KV, DIM, PAGE, BEAMS, BATCH, VOCAB = 4, 2, 64, 16, 3, 5, 4100
SLOTS, STRIDE, PAGES = BATCH * BEAMS, 30, 1000


class Step:
    """Buffers and argument blocks of a step: `new` tokens a slot behind lengths of 20 to 300."""

    def __init__(self, torch, mtp, new, lse_given):
        self.torch, self.mtp, self.new = torch, mtp, new
        gen = torch.Generator(device="cuda").manual_seed(11)
        i32 = dict(dtype=torch.int32, device="cuda")
        lens = [20 + 19 * (s // BEAMS) + new for s in range(SLOTS)]
        order = torch.randperm(PAGES, generator=torch.Generator().manual_seed(4)).tolist()
        table = [[order.pop() for _ in range(-(-(n - new) // PAGE))] for n in lens]
        self.refs = torch.zeros(PAGES, **i32)
        self.refs[[p for t in table for p in t]] = 1
        self.table = torch.tensor([t + [-1] * (STRIDE - len(t)) for t in table], **i32)
        self.before = torch.tensor([n - new for n in lens], **i32)
        self.add = torch.full((SLOTS,), new, **i32)
        self.pool = torch.randn(PAGES, 2, 2, KV, PAGE, DIM, device="cuda", generator=gen).bfloat16()
        self.start = [t.clone() for t in (self.refs, self.table, self.pool)]
        rows = SLOTS * new
        self.x = torch.zeros(rows, HEADS + 2 * KV, DIM, dtype=torch.bfloat16, device="cuda")
        self.xs = [torch.randn(self.x.shape, device="cuda", generator=gen).bfloat16() for _ in range(4)]
        self.logits = torch.zeros(BATCH, BEAMS, VOCAB, device="cuda")
        self.ls = [torch.randn(self.logits.shape, device="cuda", generator=gen) for _ in range(4)]
        self.lse = torch.zeros(BATCH, BEAMS, device="cuda") if lse_given else None
        self.scores = torch.randn(BATCH, BEAMS, device="cuda", generator=gen)
        self.lens, self.refs2 = torch.zeros(SLOTS, **i32), torch.zeros(PAGES, **i32)
        self.cu, self.status = torch.zeros(SLOTS + 1, **i32), torch.zeros(4, **i32)
        self.places = torch.zeros(rows, dtype=torch.int64, device="cuda")
        seq, pos = torch.zeros(rows, **i32), torch.zeros(rows, **i32)
        self.out = torch.zeros(rows, HEADS, DIM, dtype=torch.bfloat16, device="cuda")
        self.out_lse = torch.zeros(rows, HEADS, device="cuda")
        self.best, self.parent, self.token = torch.zeros(BATCH, BEAMS, device="cuda"), torch.zeros(BATCH, BEAMS, **i32), torch.zeros(BATCH, BEAMS, **i32)
        self.table2, self.lens2 = torch.zeros(SLOTS, STRIDE, **i32), torch.zeros(SLOTS, **i32)
        self.refs3, self.status2 = torch.zeros(PAGES, **i32), torch.zeros(4, **i32)
        plan = mtp.page_plan_args(kv_lens=self.before, new_lens=self.add, block_table=self.table, page_refs=self.refs,
                                  out_kv_lens=self.lens, out_page_refs=self.refs2, out_cu_rows=self.cu,
                                  out_slot_map=self.places, out_row_seq=seq, out_row_pos=pos, out_status=self.status,
                                  page_size=PAGE)
        append = mtp.cache_append_args(k=self.x[:, HEADS:HEADS + KV], v=self.x[:, HEADS + KV:], slot_map=self.places,
                                       kv_pool=self.pool, layer=1)
        attend = mtp.chunk_attention_args(q=self.x[:, :HEADS], kv_pool=self.pool, layer=1, block_table=self.table,
                                          cu_rows=self.cu, kv_lens=self.lens, out=self.out, out_lse=self.out_lse,
                                          scale=0.125, max_new=new, max_keys=max(lens))
        select = mtp.beam_select_args(logits=self.logits, lse=self.lse, scores=self.scores, k=BEAMS, out_scores=self.best,
                                      out_parent=self.parent, out_token=self.token)
        reorder = mtp.beam_reorder_args(parent=self.parent, block_table=self.table, kv_lens=self.lens, page_refs=self.refs2,
                                        kv_pool=self.pool, out_block_table=self.table2, out_kv_lens=self.lens2,
                                        out_page_refs=self.refs3, out_status=self.status2)
        self.keep = (seq, pos)
        ws = [(n, torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")) for n in
              (mtp.mtp_chunk_attention_workspace_bytes(attend), mtp.mtp_beam_select_workspace_bytes(select),
               mtp.mtp_beam_reorder_workspace_bytes(reorder))]
        self.plan = lambda s: mtp.mtp_page_plan(plan, s)
        self.append = lambda s: mtp.mtp_cache_append(append, s)
        self.attend = lambda s: mtp.mtp_chunk_attention(attend, ws[0][1], ws[0][0], s)
        self.select = lambda s: mtp.mtp_beam_select(select, ws[1][1], ws[1][0], s)
        self.reorder = lambda s: mtp.mtp_beam_reorder(reorder, ws[2][1], ws[2][0], s)

    def reset(self):
        for t, was in zip((self.refs, self.table, self.pool), self.start):
            t.copy_(was)

    def feed(self, i):
        self.x.copy_(self.xs[i % 4])
        self.logits.copy_(self.ls[i % 4])
        if self.lse is not None:
            self.lse.copy_(self.torch.logsumexp(self.logits, -1))

    def results(self):
        return [t.clone() for t in (self.status, self.lens, self.table, self.places, self.out, self.out_lse, self.best, self.parent,
                                    self.token, self.table2, self.lens2, self.refs3, self.status2, self.pool)]


def same(torch, a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("new,lse_given", [(1, True), (1, False), (12, True), (60, False)])
def test_calls_behind_what_writes_their_inputs(new, lse_given):
    torch = pytest.importorskip("torch")
    st = Step(torch, lib_module(), new, lse_given)
    stream = torch.cuda.Stream()

    def run(wait):
        got = []
        with torch.cuda.stream(stream):
            for i in range(12):
                st.reset()
                torch.cuda._sleep(20000)
                st.feed(i)
                for call in (st.plan, st.append, st.attend, st.select, st.reorder):
                    call(stream)
                    if wait:
                        stream.synchronize()
                got.append(st.results())
        stream.synchronize()
        return got
    want, got = run(True), run(False)
    assert want[0][0][0] == 0 and want[0][12][0] == 0
    assert not torch.equal(want[0][4], want[1][4])
    for a, b in zip(want, got):
        assert same(torch, a, b)


@pytest.mark.parametrize("new", [1, 60])
def test_branches_of_a_graph(new):
    """Captured with a fill before them, on two branches that meet: replays equal the same calls one by one."""
    torch = pytest.importorskip("torch")
    st = Step(torch, lib_module(), new, True)
    st.feed(0)
    st.reset()
    for call in (st.plan, st.append, st.attend, st.select, st.reorder):  # (what is loaded at a first call is loaded)
        call(torch.cuda.current_stream())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        st.out.zero_()
        side.wait_stream(main)
        st.plan(main)
        st.append(main)
        with torch.cuda.stream(side):
            st.select(side)
        st.attend(main)
        main.wait_stream(side)
        st.reorder(main)
    for i in range(1, 6):
        st.feed(i)
        st.reset()
        graph.replay()
        got = st.results()
        st.feed(i)
        st.reset()
        torch.cuda.synchronize()
        for call in (st.plan, st.append, st.attend, st.select, st.reorder):
            call(torch.cuda.current_stream())
            torch.cuda.synchronize()
        assert same(torch, st.results(), got)
