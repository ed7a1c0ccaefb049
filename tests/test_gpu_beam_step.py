"""Beam searches that never wait for the GPU: prompts admitted, forked into beams, and steps of lengths, slots, appends, attention,
choice and reordering, checked against histories of tokens that are attended from the beginning by the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV
from tests.table_model import Tables, choose

pytestmark = pytest.mark.gpu

L, HQ, HKV, D, VOCAB, ROOM = 2, 4, 2, 64, 5001, 8
PROMPTS, BEAMS, BLOCKS, WIDTH, TOP = (300, 511, 40), 3, 40, 4, 4 * 256
ROWS = len(PROMPTS) * BEAMS
SCALE = 0.3


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Search:
    """A toy model (rows of K, V, Q and logits' factors per token) around the library's calls; every buffer is made once."""

    def __init__(self, seed, prefix_call):
        rng = np.random.default_rng(seed)
        half = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float16)).to(DEV)  # noqa: E731
        self.spec, self.prefix_call = b.make_spec(L, HQ, HKV, D), prefix_call
        self.kp, self.vp = (b.Pool(self.spec, D, BLOCKS, DEV, poison=True) for _ in range(2))
        self.tables = b.BlockTables(ROWS, WIDTH, BLOCKS)
        self.k_of, self.v_of, self.q_of = half(L, VOCAB, HKV, D), half(L, VOCAB, HKV, D), half(L, VOCAB, HQ, D)
        self.mix = torch.from_numpy(rng.standard_normal((3, VOCAB)).astype(np.float32) * 4).to(DEV)
        self.prompt = [rng.integers(0, VOCAB, n).tolist() for n in PROMPTS]
        self.map, self.work = b.TokenMap(self.tables, ROWS + ROOM), b.q4kv_tables_workspace(self.tables)
        self.bounds = ints([BEAMS * g for g in range(len(PROMPTS) + 1)])
        self.shared = ints([n // 256 * 256 for n in PROMPTS])
        self.last = torch.zeros(ROWS, dtype=torch.int32, device=DEV)
        self.score = torch.full((ROWS,), -float("inf"), device=DEV)
        self.end = torch.full((ROWS,), -1, dtype=torch.int32, device=DEV)
        self.choice = b.BeamChoice(len(PROMPTS), BEAMS)
        self.logits = torch.zeros((ROWS, VOCAB), device=DEV)
        self.choose_work = b.q4kv_beam_select_workspace(self.logits, BEAMS)
        self.out = torch.empty((L, ROWS, 1, HQ, D), dtype=torch.float16, device=DEV)
        self.attend_work = torch.empty(max(b.q4kv_shared_prefix_workspace_bytes(self.spec, ROWS, TOP, L),
                                           b.q4kv_attention_workspace_bytes(self.spec, ROWS, 1, TOP, 0, L)), dtype=torch.uint8, device=DEV)

    def admit(self):
        """Prompts but for their last token, one row each; then a row per beam."""
        lens = [0] * ROWS
        for g, p in enumerate(self.prompt):
            lens[BEAMS * g] = len(p) - 1
        tokens = ints(sum((p[:-1] for p in self.prompt), []) + [0] * ROOM).long()
        places = b.TokenMap(self.tables, len(tokens))
        b.q4kv_resize_tables(self.tables, ints(lens), out=places, spec=self.spec, kpool=self.kp, vpool=self.vp, workspace=self.work)
        b.q4kv_append_slots(self.spec, self.kp, self.vp, self.k_of[:, tokens], self.v_of[:, tokens], places.slot)
        b.q4kv_beam_reorder(self.spec, self.kp, self.vp, self.tables, ints([r // BEAMS * BEAMS for r in range(ROWS)]), self.work)
        self.last.copy_(ints([self.prompt[r // BEAMS][-1] for r in range(ROWS)]))
        self.score.copy_(torch.tensor([0.0 if r % BEAMS == 0 else -float("inf") for r in range(ROWS)]))

    def step(self):
        t = self.tables
        b.q4kv_resize_tables(t, t.seq_len + 1, out=self.map, spec=self.spec, kpool=self.kp, vpool=self.vp, workspace=self.work)
        row = self.map.agent.clamp(min=0).long()
        token = self.last[row].long()
        b.q4kv_append_slots(self.spec, self.kp, self.vp, self.k_of[:, token], self.v_of[:, token], self.map.slot)
        q = self.q_of[:, self.last.long()].unsqueeze(2)
        if self.prefix_call:
            b.q4kv_shared_prefix_attention(self.spec, self.kp, self.vp, q, t.block_table, t.seq_len, self.bounds, self.shared, TOP, SCALE,
                                           out=self.out, workspace=self.attend_work)
        else:
            b.q4kv_batched_attention(self.spec, self.kp, self.vp, q, t.block_table, t.seq_len, TOP, SCALE, out=self.out, workspace=self.attend_work)
        h = self.out[1, :, 0, :, :].float()
        self.logits.copy_(h[:, 0, :1] * self.mix[0] + h[:, 1, 1:2] * self.mix[1] + h[:, 3, 5:6] * self.mix[2])
        self.logits[:, ::13] = -float("inf")                                    # tokens that a grammar bans
        b.q4kv_beam_select(self.logits, self.score, self.bounds, BEAMS, end_token=self.end, out=self.choice, workspace=self.choose_work)
        parent = self.choice.parent.view(-1)
        b.q4kv_beam_reorder(self.spec, self.kp, self.vp, t, parent, self.work)
        self.last.copy_(self.choice.token.view(-1))
        self.score.copy_(self.choice.score.view(-1))
        self.end.copy_(torch.where((self.last % 97 == 1) | (self.end[parent.clamp(min=0).long()] >= 0), self.last, -1))

    def all(self):
        return [self.last, self.score, self.end, self.out, self.logits, self.tables.block_table, self.tables.seq_len, self.tables.refs,
                self.tables.refused, self.map.slot, self.map.agent, self.map.position, self.map.begin, self.kp.codes, self.vp.bias]


def attended(s, history, layer_q):
    """The oracle's attention of one row: its tokens cached one after the other, the last one's query."""
    spec = oracle.make_spec(L, HQ, HKV, D, D, False)
    kp, vp = oracle.Pool(spec, D, WIDTH), oracle.Pool(spec, D, WIDTH)
    table, at = np.arange(WIDTH, dtype=np.int32)[None], torch.tensor(history, device=DEV)
    k, v = (x[:, at].cpu().numpy()[:, None] for x in (s.k_of, s.v_of))
    oracle.append(spec, kp, vp, k, v, table, np.zeros(1, np.int32))
    return oracle.attention(spec, kp, vp, layer_q[:, None, None], table, [len(history)], SCALE)[:, 0, 0]


@pytest.mark.parametrize("prefix_call", [False, True])
def test_beams_attend_to_their_own_histories(prefix_call):
    s = Search(3, prefix_call)
    s.admit()
    model = Tables(np.full((ROWS, WIDTH), -1, np.int32), [0] * ROWS, np.zeros(BLOCKS, np.int32), [])
    model.resize([len(s.prompt[r // BEAMS]) - 1 if r % BEAMS == 0 else 0 for r in range(ROWS)], 2000)
    model.reorder([r // BEAMS * BEAMS for r in range(ROWS)])
    history = [s.prompt[r // BEAMS][:-1] for r in range(ROWS)]
    parents = set()
    for step in range(9):
        last, score, end = s.last.tolist(), s.score.tolist(), s.end.tolist()
        s.step()
        torch.cuda.synchronize()
        history = [h + [t] for h, t in zip(history, last)]
        for r in range(ROWS):
            if step % 4 == 0 or r % BEAMS == step % BEAMS:
                want = attended(s, history[r], s.q_of[:, last[r]].cpu().numpy()).astype(np.float64)
                got = s.out[:, r, 0].double().cpu().numpy()
                assert (np.abs(got - want) <= 2e-3 + 2e-3 * np.abs(want)).all(), (step, r)
        parent, token, total, _ = choose(s.logits.double().cpu().numpy(), np.array(score, np.float32).astype(np.float64), s.bounds.tolist(), BEAMS, end)
        assert s.choice.parent.tolist() == parent.tolist() and s.choice.token.tolist() == token.tolist()
        parent = parent.reshape(-1).tolist()
        assert model.resize([n + 1 for n in model.len], ROWS + ROOM)[1] == s.map.slot.tolist()
        model.reorder(parent)
        assert np.array_equal(model.table, s.tables.block_table.cpu().numpy()) and np.array_equal(model.refs, s.tables.refs.cpu().numpy())
        assert s.tables.seq_len.tolist() == model.len and s.tables.refused.item() == 0
        history = [history[p] for p in parent]
        parents |= {tuple(parent)}
    assert len(parents) > 3                                                     # rows did change places


def test_a_captured_step():
    """The whole step in a graph, replayed between eager work, against the same steps called one by one."""
    eager, s = Search(5, True), Search(5, True)
    eager.admit(), s.admit()
    eager.step(), s.step()                                                      # both are where a program captures
    torch.cuda.synchronize()
    kept = [t.clone() for t in (s.last, s.score, s.end, s.tables.block_table, s.tables.seq_len, s.tables.refs, s.kp.codes, s.kp.scale, s.kp.bias,
                                s.vp.codes, s.vp.scale, s.vp.bias)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            s.step()
    torch.cuda.synchronize()
    for t, k in zip((s.last, s.score, s.end, s.tables.block_table, s.tables.seq_len, s.tables.refs, s.kp.codes, s.kp.scale, s.kp.bias,
                     s.vp.codes, s.vp.scale, s.vp.bias), kept):
        t.copy_(k)
    for step in range(6):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for got, want in zip(s.all(), eager.all()):
            assert torch.equal(got, want), step
