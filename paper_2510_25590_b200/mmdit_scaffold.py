"""Stand-in transformer stack for the sampler-loop configuration (8 random blocks in the benchmark),
run the region-aware way.  Scaffold around the library, not part of it: the paper's editors and their
weights are not available, so the blocks' dense projections, normalisations and activations are
plain torch operations on random weights (library GEMMs), while everything the method is about goes
through the C-ABI: the rotary / RMS-normalised Q, K, V rows (``fresh_qkv``), the attention of a full
step (``region_attention`` with no cache), the Region-Instruction KV cache of every block
(``rikv_store``) and the region step's attention over [fresh | cached] keys (``region_attention``).

It offers the two callbacks the sampler loop (``loop.RegionELoop``) asks of a velocity model:

    full(x, t, store)                 every row of [text | image | reference] through every block; with
                                      ``store`` the blocks' K and V are kept (Sec. 4, "Stabilization Stage")
    region(x_e, t, edit_idx, n_edit)  only the recomputed rows (edited tokens, plus the text rows under the
                                      attention equation as printed) through every block, their queries
                                      attending over their own fresh K, V and the kept K, V of all other rows

``products`` names what multiplies the rows with the weight set of their stream (text, or image and
reference): "torch", two library products and a concatenation; "grouped", one ``grouped_matmul`` with both weight
sets, the rows' ranges on the device and the activation in its epilogue; "mxfp4", the same on 4-bit operands
(weights quantised once, rows in front of each product; the modulation's single rows stay in bf16).  ``cache``
names how the blocks' kept K and V are stored between a full step and the region steps behind it: "bf16", or
"mxfp4" (4 bits, widened in front of each attention).

Outside a planted mask the velocity is replaced by the straight line to the reference latent, so that
the Adaptive Region Partition has a region to find in a stack that was never trained.  One request
(batch 1); the block definition is stated in the oracle's counterpart of this file.
"""
from __future__ import annotations

from . import binding


class MMDiTScaffold:
    def __init__(self, weights, n_text, n_img, n_ref, heads, head_dim, blocks, cos, sin, ref, planted,
                 membership=binding.ROWS_PAPER, products="torch", cache="bf16"):
        import torch
        if products not in ("torch", "grouped", "mxfp4") or cache not in ("bf16", "mxfp4"):
            raise binding.RegionEError(f"no products {products!r} or cache {cache!r}")
        self.products, self.cache = products, cache
        self.w = weights                                   # name -> bf16 CUDA tensor
        self.n_text, self.n_img, self.n_ref = n_text, n_img, n_ref
        self.n_full = n_text + n_img + n_ref
        self.H, self.D, self.L, self.hidden = heads, head_dim, blocks, heads * head_dim
        self.cos, self.sin, self.ref, self.planted = cos, sin, ref, planted
        self.membership = membership
        self.loop = None
        dev, i32, bf = ref.device, torch.int32, torch.bfloat16
        n, H, D = self.n_full, heads, head_dim
        buf = lambda rows: torch.empty((1, rows, H, D), dtype=bf, device=dev)
        self.k_full = [buf(n) for _ in range(blocks)]       # K, V of every row at the last storing step
        self.v_full = [buf(n) for _ in range(blocks)]
        # the rows a region step does not recompute: of every block, or codes of every block and one block's widened
        self.k_cache = [buf(n) for _ in range(blocks if cache == "bf16" else 1)]
        self.v_cache = [buf(n) for _ in range(blocks if cache == "bf16" else 1)]
        if cache == "mxfp4":
            bits = lambda d: torch.empty((1, n, H, D // d), dtype=torch.uint8, device=dev)
            self.codes = [(bits(2), bits(2), bits(32), bits(32)) for _ in range(blocks)]
        self.scratch = [buf(n) for _ in range(5)]
        self.all_rows = torch.arange(n, dtype=i32, device=dev).view(1, n)
        self.n_all = torch.tensor([n], dtype=i32, device=dev)
        self.zero = torch.zeros(1, dtype=i32, device=dev)
        self.query_rows = torch.zeros((1, n), dtype=i32, device=dev)
        self.cache_rows = torch.zeros((1, n), dtype=i32, device=dev)
        self.n_query, self.n_cache = torch.zeros(1, dtype=i32, device=dev), torch.zeros(1, dtype=i32, device=dev)
        self.dev_status = torch.zeros(1, dtype=i32, device=dev)
        ws = binding.region_attention_workspace(1, n, n, n, H, D)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)
        self._stale = True                                   # row lists / compacted caches need rebuilding
        self._nq = 0
        self.library_launches = 0
        if products != "torch":
            self._lay_out_weights()

    def bind(self, loop):
        """The loop whose partition lists (keep_idx) the region steps read."""
        self.loop = loop
        return self

    # ---- torch pieces (scaffold) ----------------------------------------------------------
    def _ln(self, h):
        import torch
        return torch.nn.functional.layer_norm(h.float(), (self.hidden,), eps=1e-6)

    # ---- products of both streams in one call ------------------------------------------------
    def _lay_out_weights(self):
        """Both streams' weights of a product as [2, N, K] (codes and scales with 4-bit products), once."""
        import torch
        hd, dev, i32 = self.hidden, self.ref.device, torch.int32
        self.sets = {}
        for l in range(self.L):
            for name in (f"q{l}", f"k{l}", f"v{l}", f"o{l}", f"fc1_{l}", f"fc2_{l}", f"mod{l}"):
                if name[0] in "qkv":
                    j = "qkv".index(name[0])
                    both = [self.w[f"qkv{l}_{s}"][:, j * hd:(j + 1) * hd] for s in (0, 1)]
                else:
                    both = [self.w[f"{name}_{s}"] for s in (0, 1)]
                w = torch.stack([b.T.contiguous() for b in both])
                if self.products == "mxfp4" and not name.startswith("mod"):
                    codes = torch.empty((2, w.shape[1], w.shape[2] // 2), dtype=torch.uint8, device=dev)
                    scales = torch.empty((2, w.shape[1], w.shape[2] // 32), dtype=torch.uint8, device=dev)
                    binding.mxfp4_quantize(w, codes, scales, dev_status=self.dev_status)
                    w = (codes, scales)
                self.sets[name] = w
        ints = lambda *v: torch.tensor(v, dtype=i32, device=dev)
        self.one_each = ints(0, 1), ints(1, 2)               # the modulation's rows: one per stream
        self.full_ranges = ints(0, self.n_text), ints(self.n_text, self.n_full)
        self.region_begin, self.region_end = ints(0, 0), ints(0, 0)

    def _operand(self, a):
        """Rows as a product of ``products`` takes them."""
        import torch
        if self.products != "mxfp4":
            return a
        rows, K = a.shape
        codes = torch.empty((1, rows, K // 2), dtype=torch.uint8, device=a.device)
        scales = torch.empty((1, rows, K // 32), dtype=torch.uint8, device=a.device)
        binding.mxfp4_quantize(a[None], codes, scales, dev_status=self.dev_status)
        self.library_launches += 1
        return codes[0], scales[0]

    def _product(self, operand, name, ranges, out, activation=binding.ACT_NONE):
        """out[r] = act(rows times the weight set of their range's stream)."""
        w = self.sets[name]
        if isinstance(w, tuple):
            binding.mxfp4_grouped_matmul(*operand, *w, *ranges, out, activation=activation, dev_status=self.dev_status)
        else:
            binding.grouped_matmul(operand, w, *ranges, out, activation=activation, dev_status=self.dev_status)
        self.library_launches += 1
        return out

    def _mm(self, a, name, n_text_rows, activation=binding.ACT_NONE):
        """Rows [text | others] times the weight set of their stream."""
        import torch
        if self.products != "torch":
            w = self.sets[name]
            out = torch.empty((a.shape[0], (w[0] if isinstance(w, tuple) else w).shape[1]), dtype=torch.bfloat16, device=a.device)
            return self._product(self._operand(a), name, self.ranges, out, activation)
        if activation == binding.ACT_GELU_TANH:
            return torch.nn.functional.gelu(self._mm(a, name, n_text_rows), approximate="tanh")
        w0, w1 = self.w[f"{name}_0"], self.w[f"{name}_1"]
        if n_text_rows == 0:
            return a @ w1
        return torch.cat([a[:n_text_rows] @ w0, a[n_text_rows:] @ w1])

    def _mods(self, t, l, n_text_rows, rows):
        import torch
        c = torch.tanh(t * self.w["t_a"].float() + self.w["t_b"].float()).to(torch.bfloat16)[None]
        if self.products != "torch":
            both = torch.empty((2, 6 * self.hidden), dtype=torch.bfloat16, device=c.device)
            m = self._product(c.expand(2, -1).contiguous(), f"mod{l}", self.one_each, both).float().split(1)
        else:
            m = [(c @ self.w[f"mod{l}_{s}"]).float() for s in (0, 1)]           # [1, 6 * hidden] per stream
        full = torch.cat([m[0].expand(n_text_rows, -1), m[1].expand(rows - n_text_rows, -1)])
        return full.chunk(6, dim=-1)

    def _blocks(self, h, t, positions, n_rows_dev, n_text_rows, attend, keep_kv):
        import torch
        bf = torch.bfloat16
        rows, H, D, hd = h.shape[0], self.H, self.D, self.hidden
        q_s, k_s, v_s, q_d, o_d = self.scratch              # each [1, rows, H, D]
        for l in range(self.L):
            sh1, sc1, g1, sh2, sc2, g2 = self._mods(t, l, n_text_rows, rows)
            a = (self._ln(h) * (1.0 + sc1) + sh1).to(bf)
            wq = lambda s: self.w[f"qkv{l}_{s}"]
            operand = None if self.products == "torch" else self._operand(a)
            for j, dst in enumerate((q_s, k_s, v_s)):            # three projections, each into its own buffer
                out = dst.view(-1, hd)[:rows]
                if operand is not None:
                    self._product(operand, f"{'qkv'[j]}{l}", self.ranges, out)
                    continue
                if n_text_rows:
                    torch.matmul(a[:n_text_rows], wq(0)[:, j * hd:(j + 1) * hd], out=out[:n_text_rows])
                torch.matmul(a[n_text_rows:], wq(1)[:, j * hd:(j + 1) * hd], out=out[n_text_rows:])
            k_d, v_d = (self.k_full[l], self.v_full[l]) if keep_kv else (self._tmp("_ktmp", rows), self._tmp("_vtmp", rows))
            binding.fresh_qkv(q_s, k_s, v_s, positions, n_rows_dev,
                              self.w[f"qn{l}"], self.w[f"kn{l}"], 1e-6, self.cos, self.sin, binding.ROPE_INTERLEAVED,
                              q_d, k_d, v_d, src_compact=True, dev_status=self.dev_status)
            self.library_launches += 1
            attend(l, q_d, k_d, v_d, o_d)
            o = o_d.view(-1, hd)[:rows]
            h = (h.float() + g1 * self._mm(o, f"o{l}", n_text_rows).float()).to(bf)
            m = (self._ln(h) * (1.0 + sc2) + sh2).to(bf)
            u = self._mm(m, f"fc1_{l}", n_text_rows, binding.ACT_GELU_TANH)
            h = (h.float() + g2 * self._mm(u, f"fc2_{l}", n_text_rows).float()).to(bf)
        return h

    def _tmp(self, name, rows):
        import torch
        t = getattr(self, name, None)
        if t is None or t.shape[1] != rows:
            t = torch.empty((1, rows, self.H, self.D), dtype=torch.bfloat16, device=self.ref.device)
            setattr(self, name, t)
        return t

    def _blend(self, v_net, x_rows, ref_rows, planted_rows, t):
        import torch
        line = ((x_rows.float() - ref_rows.float()) / t).to(torch.bfloat16)
        return torch.where(planted_rows[:, None], v_net, line)

    # ---- the two calls of the loop ----------------------------------------------------------
    def full(self, x, t, store):
        import torch
        if isinstance(t, (list, tuple)):
            t, store = t[0], store[0]
        w = self.w
        emb = lambda z: z[0] @ w["w_in"] + w["b_in"]
        h = torch.cat([w["text_emb"], emb(x), emb(self.ref) + w["ref_emb"]])

        def attend(l, q, k, v, o):
            binding.region_attention(q, k, v, None, None, self.n_all, self.n_all, self.zero, o,
                                     workspace=self.workspace, dev_status=self.dev_status)
            self.library_launches += 2

        if self.products != "torch":
            self.ranges = self.full_ranges
        # (the scratch buffers span the whole sequence here, so no slicing copies happen)
        h = self._blocks(h, float(t), self.all_rows, self.n_all, self.n_text, attend, keep_kv=bool(store))
        if store:
            self._stale = True
        v_net = (self._ln(h[self.n_text:self.n_text + self.n_img]).to(torch.bfloat16) @ w["w_out"])
        return self._blend(v_net, x[0], self.ref[0], self.planted[0], float(t))[None]

    def _refresh_lists_and_caches(self, edit_idx, n_edit):
        lp = self.loop
        binding.region_rows(edit_idx, lp.keep_idx, n_edit, self.n_text, self.n_ref, self.membership,
                            self.query_rows, self.n_query, self.cache_rows, self.n_cache, dev_status=self.dev_status)
        for l in range(self.L):
            if self.cache == "mxfp4":
                binding.rikv_store_mxfp4(self.k_full[l], self.v_full[l], self.cache_rows, self.n_cache, *self.codes[l],
                                         dev_status=self.dev_status)
            else:
                binding.rikv_store(self.k_full[l], self.v_full[l], self.cache_rows, self.n_cache, self.k_cache[l],
                                   self.v_cache[l], dev_status=self.dev_status)
        self.library_launches += 1 + self.L
        self._nq = int(self.n_query.item())                  # one host read per run of region steps: the GEMM sizes
        self._stale = False

    def region(self, x_e, t, edit_idx, n_edit):
        import torch
        if isinstance(t, (list, tuple)):
            t = t[0]
        if self._stale:
            self._refresh_lists_and_caches(edit_idx, n_edit)
        w, nq = self.w, self._nq
        with_text = self.membership == binding.ROWS_PAPER
        nt = self.n_text if with_text else 0
        ne = nq - nt
        h = x_e[0, :ne] @ w["w_in"] + w["b_in"]
        if with_text:
            h = torch.cat([w["text_emb"], h])
        positions = self.query_rows[:, :nq].contiguous()
        if self.products != "torch":                         # text rows [0, nt), the others [nt, n_query)
            self.region_begin[1:].fill_(nt)
            self.region_end[:1].fill_(nt)
            self.region_end[1:].copy_(self.n_query)
            self.ranges = self.region_begin, self.region_end

        def attend(l, q, k, v, o):
            at = l
            if self.cache == "mxfp4":
                at = 0
                binding.rikv_load_mxfp4(*self.codes[l], self.n_cache, self.k_cache[0], self.v_cache[0], dev_status=self.dev_status)
                self.library_launches += 1
            binding.region_attention(q, k, v, self.k_cache[at], self.v_cache[at], self.n_query, self.n_query,
                                     self.n_cache, o, workspace=self.workspace, dev_status=self.dev_status)
            self.library_launches += 2

        h = self._blocks_compact(h, float(t), positions, nt, attend)
        v_net = (self._ln(h[nt:]).to(torch.bfloat16) @ w["w_out"])
        e = edit_idx[0, :ne].long()
        out = torch.zeros_like(x_e)
        out[0, :ne] = self._blend(v_net, x_e[0, :ne], self.ref[0, e], self.planted[0, e], float(t))
        return out

    def _blocks_compact(self, h, t, positions, n_text_rows, attend):
        """The same blocks over a compact set of rows (own buffers of that size)."""
        rows = h.shape[0]
        saved = self.scratch
        self.scratch = [self._tmp(f"_c{i}", rows) for i in range(5)]
        try:
            return self._blocks(h, t, positions, self.n_query, n_text_rows, attend, keep_kv=False)
        finally:
            self.scratch = saved
